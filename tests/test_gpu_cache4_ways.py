"""Which way attention over 4 bits goes, and that each is as near as its own roundings allow."""

import pytest
import torch

from tests.test_gpu_cache4 import _attend, _close, _gmc, _h, _lib  # noqa: F401

pytestmark = pytest.mark.gpu

WAYS = [
    # lens, tokens of each, H, Hkv, d, page, window, sinks, launches, way
    ([130, 200, 90], 9, 14, 2, 128, 32, 0, 0, 1, "codes"),
    ([130, 200, 90], 9, 14, 2, 64, 8, 64, 3, 1, "codes"),
    ([700] * 6, 150, 14, 2, 128, 64, 0, 0, 1, "codes"),
    ([1900], 12, 14, 2, 128, 32, 0, 0, 2, "codes"),              # in parts, joined
    ([2000], 5, 4, 2, 64, 64, 900, 40, 2, "codes"),
    ([900, 865], 3, 100, 1, 128, 16, 200, 33, 2, "codes"),       # a tile a token
    ([300, 200, 201, 256, 257] * 2 + [300] * 2, 200, 8, 4, 64, 16, 0, 0, 2, "unpacked"),
    ([300, 200, 201, 256, 257] * 2 + [300] * 2, 200, 8, 4, 64, 7, 40, 3, 2, "unpacked"),
    ([700] * 6, 450, 14, 2, 128, 48, 0, 0, 2, "unpacked"),
    ([700] * 6, 450, 14, 2, 128, 64, 250, 130, 2, "unpacked"),
    ([257] * 8, 257, 2, 1, 256, 16, 0, 0, 3, "unpacked"),        # in parts, joined
    ([1], 1, 1, 1, 256, 16, 0, 0, 1, "decode"),
    ([700, 40, 33, 12], 9, 8, 2, 256, 48, 0, 0, 2, "alone"),     # token by token
    ([900, 64], 40, 11, 1, 256, 16, 100, 33, 3, "alone"),        # 8 query heads a launch
    ([500, 1, 2000], 1, 14, 2, 128, 64, 0, 0, 2, "decode"),      # in stretches, joined
]


def _way(c, cap, T, ws):
    """What the workspace, filled with -1 before, says: the unpacked rows' pages in order, or
    each token's length, lie at its start."""
    n = c.B * -(-cap // 128)
    if torch.equal(ws[:n].cpu(), torch.arange(n, dtype=torch.int32)):
        return "unpacked"
    lens = [n - T + t + 1 for n in c.lens for t in range(T)]
    if c.d == 256 and T > 1 and ws[:len(lens)].tolist() == lens:
        return "alone"
    return "decode" if T == 1 else "codes"


@pytest.mark.parametrize("lens,T,H,Hkv,d,page,window,sinks,launches,way", WAYS)
def test_attend_goes_its_way(lens, T, H, Hkv, d, page, window, sinks, launches, way):
    from tests import cache_harness as A
    C, gmc = _h(), _gmc()
    c = C.Case4(lens, H, Hkv, d, page, [T] * len(lens), spread=2.0)
    cap = min(max(lens) + 1, c.table.shape[1] * page)
    cache, q = c.cache(max_len=cap), c.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(len(q), H, device="cuda")
    size = gmc.attend_workspace_size(cache, H, T)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    before = gmc.launch_count()
    gmc.attend(cache, q, out, T, window=window, sinks=sinks, lse=lse, workspace=ws)
    count = gmc.launch_count() - before
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    assert _way(c, cap, T, ws[:size // 4 * 4].view(torch.int32)) == way and count == launches
    for b, n in enumerate(lens):
        small = 2.0 ** -32 * c.V[b].double().abs().sum(0).repeat_interleave(H // Hkv, 0)
        for x in {0, 1, T - 1, *range(b, T, 1 + T // 16)} & set(range(T)):
            at = b * T + x
            ref, z, _, bound, s = A.attention(c.K[b], c.V[b], c.q[at], n - T + x, window, sinks)
            if way == "unpacked":  # the tensor cores' way rounds weights to bf16
                tol = A.tolerance(c.dt, d, s, roundings=2 if d < 256 else 1)
            else:
                tol = C.tolerance(c, s)
            _close(out[at], ref, bound + small / tol, tol, f"sequence {b}, new token {x}")
            _close(lse[at], z, torch.ones_like(z), A.lse_tolerance(d, s) * 4, "lse")


@pytest.mark.parametrize("which", ["k", "v", "both"])
@pytest.mark.parametrize("lens,news,H,Hkv,d", [([300] * 12, [200] * 12, 8, 4, 64),   # unpacked
                                               ([700] * 6, [450] * 6, 14, 2, 128),
                                               ([257] * 8, [257] * 8, 2, 1, 256),
                                               ([90, 70], [5, 3], 4, 2, 256)])       # alone
def test_nan_reaches_the_rows_that_see_it(lens, news, H, Hkv, d, which):
    c = _h().Case4(lens, H, Hkv, d, 16, news)
    plain, _ = _attend(c, 0, 0)
    bad, t = lens[0] - 4, news[0]  # of the first sequence: its last four new tokens see it
    for pool, n in ((c.pool_k, "k"), (c.pool_v, "v")):
        if which in (n, "both"):
            for x in c.halves(pool):
                x[int(c.table[0, bad // c.page]), :, bad % c.page] = 0xf9
    out, _ = _attend(c, 0, 0)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    assert bool(torch.isnan(out[t - 4:t]).all()) and torch.equal(out[t:], plain[t:])
    # rows computed one by one: each within its roundings of the same row of values
    a, b = out[:t - 4].double(), plain[:t - 4].double()
    assert bool(torch.isfinite(a).all())
    assert float((a - b).abs().max()) <= 2 * 2.0 ** -8 * float(b.abs().max())
