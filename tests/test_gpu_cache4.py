"""The cache held in 4 bits on the GPU: packing, reading, decode, attend and evict against their
definitions in 64 bits."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _h():
    from tests import cache4_harness as C
    return C


def _gmc():
    from paper_2608_02134_gb300 import gmc
    return gmc


def _close(got, want, bound, tol, what):
    got = got.double().cpu()
    err = (got - want).abs()
    limit = tol * bound + 1e-30
    bad = ~(err <= limit)
    assert not bool(bad.any()), \
        f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / limit).max()):.3g} x"


# ---- packing -----------------------------------------------------------------------------
def _hard_rows(d):
    """Rows [n, d] of bf16: ties of every scale and level, the range's ends, what is not finite."""
    C = _h()
    rows = []
    for m in list(range(8, 16)):
        for e in (-10, 0, 7):
            s = m / 8 * 2.0 ** e
            ties = [(a + b) / 2 * s for a, b in zip(C.LEVELS, C.LEVELS[1:])]
            rows.append([6 * s] + ties + [-x for x in ties] + [0.0])
    for m in range(1, 8):  # scales below the smallest normal half
        s = m * 2.0 ** -17
        ties = [(a + b) / 2 * s for a, b in zip(C.LEVELS, C.LEVELS[1:])]
        rows.append([-6 * s] + ties + [-x for x in ties] + [-0.0])
    # ties of the scale itself: 6 times the middle between two scales
    for b in list(range(1, 40)) + [100, 101, 0xdf]:
        rows.append([6 * (C.SCALES[b] + C.SCALES[b + 1]) / 2, 1.0 * C.SCALES[b]] + [0.0] * 14)
    for x in (0.0, 1e-39, 1e-6, 2.0 ** -18 * 6, 4e4, 49152.0, 5e4, 7e4, 3e38):
        rows.append([x, -x / 2, x / 3, -x / 5] + [x / 7] * 12)
    for x in (math.inf, -math.inf, math.nan):
        rows.append([1.0] * 7 + [x] + [2.0] * 8)
    blocks = torch.tensor(rows, dtype=torch.float64).bfloat16()
    g = torch.Generator().manual_seed(7)
    more = -len(blocks) % (d // 16) + 3 * (d // 16)
    blocks = torch.cat([blocks, torch.randn(more, 16, generator=g).bfloat16()])
    return blocks.reshape(-1, d)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_append_packs_as_defined_and_read_gives_the_values(d):
    C, gmc = _h(), _gmc()
    x = _hard_rows(d)
    n = len(x)
    c = C.Case4([n + 3], 1, 1, d, 16, [n])
    cache = c.cache()
    k, v = x[:, None].cuda(), x.flip(0)[:, None].contiguous().cuda()
    gmc.cache_append(cache, k, v, n)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    gmc.cache_read(cache, ko, vo, n)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    for raw, pool, out in ((k, c.dk, ko), (v, c.dv, vo)):
        want = C.pack(raw.cpu())
        C.same_rows(c.rows(pool.cpu(), 0, range(3, n + 3)), want, "packed")
        got, ref = out.cpu().double(), C.unpack(*want)
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(got.nan_to_num(), ref.nan_to_num())
    # what was there before stays
    C.same_rows(c.rows(c.dk.cpu(), 0, range(3)), C.pack(c.raw_K[0][:3]), "earlier rows")


@pytest.mark.parametrize("lens,news,Hkv,d,page,pad", [
    ([1], [1], 1, 64, 1, 0), ([40, 7, 200], [40, 1, 130], 2, 128, 16, 32),
    ([65, 64], [65, 3], 3, 64, 7, 0), ([300], [90], 1, 256, 48, 16),
    ([20, 30, 5], [0, 30, 2], 4, 128, 16, 0)])
@pytest.mark.parametrize("packed", [False, True])
def test_append_and_read_ragged(lens, news, Hkv, d, page, pad, packed):
    """Rows of no sequence, slots of nobody and pages' padding are left as they were."""
    C, gmc = _h(), _gmc()
    c = C.Case4(lens, Hkv, Hkv, d, page, news, pad=pad)
    for b in range(c.B):
        for j in range(lens[b] - news[b], lens[b]):
            c.blank(b, j)
    cache = c.cache()
    k = torch.cat([x[n - t:] for x, n, t in zip(c.raw_K, lens, news)])
    v = torch.cat([x[n - t:] for x, n, t in zip(c.raw_V, lens, news)])
    if packed:
        kv, at = [], 0
        for t in news:
            kv += [k[at:at + t], v[at:at + t]]
            at += t
        gmc.cache_append(cache, torch.cat(kv).cuda(), None, max(news), offsets=c.offsets())
    else:
        gmc.cache_append(cache, k.cuda(), v.cuda(), max(news), offsets=c.offsets())
    ko = torch.full((len(k) + 2, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    vo = torch.full_like(ko, 7.0)
    gmc.cache_read(cache, ko, vo, max(news), offsets=c.offsets())
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    whole = C.Case4(lens, Hkv, Hkv, d, page, news, pad=pad)  # all rows in place
    for got, want in ((c.dk, whole.pool_k), (c.dv, whole.pool_v)):
        a, b = c.halves(got.cpu()), c.halves(want)
        C.same_rows(a, b, "pool")
        n = page * d * 9 // 16
        assert torch.equal(got.cpu()[..., n:], want[..., n:])
    for got, raw in ((ko, k), (vo, v)):
        assert torch.equal(got[:len(k)].cpu().double(), C.unpack(*C.pack(raw)))
        assert bool((got[len(k):] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_of_other_caches(dtype):
    from tests.cache_harness import Case
    gmc = _gmc()
    for layout in ("heads", "slots"):
        c = Case([70, 33, 5], 2, 2, 80, dtype, 16, [70, 4, 0], layout=layout)
        cache = c.cache()
        k = torch.full((76, 2, 80), 7.0, dtype=c.dt, device="cuda")
        v = torch.full_like(k, 7.0)
        gmc.cache_read(cache, k, v, 70, offsets=c.offsets())
        torch.cuda.synchronize()
        for got, rows in ((k, c.K), (v, c.V)):
            want = torch.cat([x[n - t:] for x, n, t in zip(rows, c.lens, c.news)])
            assert torch.equal(got[:74].cpu(), want) and bool((got[74:] == 7.0).all())


def test_read_into_rows_of_16_byte_alignment():
    C, gmc = _h(), _gmc()
    c = C.Case4([50], 1, 1, 64, 16)
    cache = c.cache()
    room = torch.empty(2 * 50 * 64 + 32, dtype=torch.bfloat16, device="cuda")
    k, v = (room[8 + i * 50 * 64:][:50 * 64].reshape(50, 1, 64) for i in range(2))
    gmc.cache_read(cache, k, v, 50)
    torch.cuda.synchronize()
    assert k.data_ptr() % 32 == 16
    assert torch.equal(k.cpu(), c.K[0]) and torch.equal(v.cpu(), c.V[0])


def test_read_leaves_rows_it_cannot_find():
    C, gmc = _h(), _gmc()
    c = C.Case4([5], 1, 1, 64, 16)
    cache = c.cache(max_len=16)
    k = torch.full((8, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, 7.0)
    gmc.cache_read(cache, k, v, 8)  # three rows before the sequence
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE
    assert bool((k[:3] == 7.0).all()) and torch.equal(k[3:, 0].cpu(), c.K[0][:, 0])
    c.table[0, 0] = 10 ** 6  # a page outside the pool
    cache = c.cache(max_len=16)
    k.fill_(7.0)
    gmc.cache_read(cache, k[:5].contiguous(), v[:5].contiguous(), 5)
    gmc.cache_append(cache, v[:5].contiguous(), v[:5].contiguous(), 5)
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE
    assert torch.equal(c.dk.cpu(), c.pool_k) and torch.equal(c.dv.cpu(), c.pool_v)


# ---- decode ------------------------------------------------------------------------------
DECODE = [
    # lens, H, Hkv, d, page, window, sinks, append, scores
    ([1], 1, 1, 64, 16, 0, 0, True, True),
    ([1, 0, 2], 4, 2, 128, 16, 0, 0, False, True),
    ([31, 32, 33, 64], 8, 1, 128, 16, 0, 0, True, True),
    ([322], 28, 4, 128, 16, 0, 0, True, True),
    ([322], 28, 4, 128, 16, 0, 0, False, False),
    ([700, 5, 129], 12, 2, 64, 48, 0, 0, True, True),
    ([700, 5, 129], 6, 2, 256, 7, 0, 0, True, True),
    ([2085, 300, 999, 1], 28, 4, 128, 64, 0, 0, True, True),
    ([1999], 4, 4, 128, 64, 0, 0, False, False),
    ([1999], 16, 1, 64, 64, 300, 17, True, True),
    ([1500, 40], 11, 1, 256, 32, 64, 3, True, True),
    ([600], 40, 1, 128, 128, 1, 0, True, True),
    ([700, 90], 18, 2, 128, 16, 0, 0, True, True),
    ([700, 90], 32, 2, 128, 64, 100, 5, False, True),
    ([500, 33, 64], 26, 2, 64, 16, 0, 0, True, True),
    ([600, 599], 3, 3, 64, 16, 33, 0, False, True),
    ([6000], 2, 1, 128, 256, 0, 0, False, True),
    ([5000, 1, 2500], 7, 1, 64, 64, 4096, 4, True, False),
]


def _decode(c, window, sinks, append, scores, max_len=None, **kw):
    gmc = _gmc()
    if append:
        for b, n in enumerate(c.lens):
            if n and int(c.table[b, (n - 1) // c.page]) < len(c.pool_k):
                c.blank(b, n - 1)
    cache = c.cache(max_len=max_len or min(max(c.lens) + 3, c.table.shape[1] * c.page))
    zero = torch.zeros(c.Hkv, c.d, dtype=torch.bfloat16)
    k = torch.stack([x[-1] if len(x) else zero for x in c.raw_K]).cuda()
    v = torch.stack([x[-1] if len(x) else zero for x in c.raw_V]).cuda()
    places = (max_len or max(c.lens)) + 5
    g = torch.Generator().manual_seed(3)
    before = torch.rand(c.B, c.Hkv, places, generator=g)
    new = torch.full((c.B, c.Hkv, places), 9.0, device="cuda")
    out = torch.full((c.B, c.H, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.B, c.H), 7.0, device="cuda")
    gmc.decode(cache, c.q.cuda(), out, k if append else None, v if append else None, window, sinks,
               lse=lse, scores=before.cuda() if scores else None,
               out_scores=new if scores else None, **kw)
    return out, lse, before, new


def _check_decode(c, window, sinks, append, scores, max_len=None):
    from tests import cache_harness as A
    C = _h()
    H, Hkv, d, G = c.H, c.Hkv, c.d, c.H // c.Hkv
    out, lse, before, new = _decode(c, window, sinks, append, scores, max_len)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    new, dk, dv = new.cpu(), c.dk.cpu(), c.dv.cpu()
    for b, n in enumerate(c.lens):
        ref, z, w, bound, size = A.attention(c.K[b], c.V[b], c.q[b], n - 1, window, sinks)
        tol = C.tolerance(c, size)
        small = 2.0 ** -25 * c.V[b].double().abs().sum(0).repeat_interleave(G, 0)  # tiny weights
        _close(out[b], ref, bound + small / tol, tol, f"sequence {b}")
        if n == 0:
            assert bool((lse[b] == -math.inf).all())
            continue
        _close(lse[b], z, torch.ones_like(z), A.lse_tolerance(d, size) * 4, "lse")
        if scores:
            old = before[b, :, :n].double()
            if append:
                old[:, n - 1] = 0.0
            got = w.reshape(Hkv, G, n).sum(1)
            _close(new[b, :, :n], old + got, old + got + 1e-6,
                   A.lse_tolerance(d, size) * 8, "scores")
            assert bool((new[b, :, n:] == 9.0).all())
        if append:
            for pool, raw in ((dk, c.raw_K), (dv, c.raw_V)):
                C.same_rows(c.rows(pool, b, [n - 1]), C.pack(raw[b][-1:]), "appended")


@pytest.mark.parametrize("lens,H,Hkv,d,page,window,sinks,append,scores", DECODE)
def test_decode_matches_its_definition(lens, H, Hkv, d, page, window, sinks, append, scores):
    c = _h().Case4(lens, H, Hkv, d, page, spread=2.0)
    _check_decode(c, window, sinks, append, scores)


@pytest.mark.parametrize("lens,H,Hkv,d,page,window,sinks,append,scores", DECODE)
def test_decode_with_room(lens, H, Hkv, d, page, window, sinks, append, scores):
    """Short sequences in a cache with room for long ones: stretches of the batch, joined."""
    width = -(-6000 // page)
    c = _h().Case4(lens, H, Hkv, d, page, spread=2.0, width=width)
    _check_decode(c, window, sinks, append, scores, max_len=width * page)


@pytest.mark.parametrize("B,H,Hkv,d,page,window,sinks,append,scores", [
    (90, 8, 4, 64, 16, 0, 0, True, True),        # two or three pairs a block
    (300, 8, 4, 64, 32, 0, 0, True, False),      # many pairs a block, runs across their borders
    (260, 6, 6, 128, 16, 0, 0, False, True),
    (200, 9, 1, 256, 48, 40, 2, True, True),     # two launches
    (64, 3, 3, 64, 7, 33, 5, True, True)])
def test_decode_of_many_sequences(B, H, Hkv, d, page, window, sinks, append, scores):
    lens = [(17 * b * b + 5 * b) % 131 for b in range(B)]  # some of none
    c = _h().Case4(lens, H, Hkv, d, page, spread=2.0)
    _check_decode(c, window, sinks, append, scores)


@pytest.mark.parametrize("window,sinks", [(2 ** 30, 3), (2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 30),
                                          (31, 32), (32, 31), (64, 64), (33, 33)])
def test_decode_windows_and_sinks_at_the_borders_of_turns(window, sinks):
    c = _h().Case4([700, 64, 65, 1], 4, 2, 128, 32, spread=2.0)
    _check_decode(c, window, sinks, True, True)


def test_decode_of_hard_queries():
    """Queries of very different sizes, zero and enormous ones: exact powers of two come out."""
    from tests import cache_harness as A
    C = _h()
    c = C.Case4([200, 77, 130, 64], 7, 1, 128, 16)
    for b, f in enumerate((0.0, 1e-30, 3e4, 1.0)):
        c.q[b] = (c.q[b].float() * f).bfloat16()
    c.q[3, :, ::3] = (c.q[3, :, ::3].float() * 2.0 ** -20).bfloat16()
    c.q[2] = (c.q[2].float() / 2.0 ** 20).bfloat16()
    out, lse, _, _ = _decode(c, 0, 0, False, False)
    torch.cuda.synchronize()
    for b, n in enumerate(c.lens):
        ref, z, w, bound, size = A.attention(c.K[b], c.V[b], c.q[b], n - 1)
        _close(out[b], ref, bound, C.tolerance(c, size) + 2.0 ** -20, f"sequence {b}")
        _close(lse[b], z, torch.ones_like(z), A.lse_tolerance(128, size) * 4, "lse")


@pytest.mark.parametrize("append", [False, True])
def test_decode_does_not_see_what_it_should_not(append):
    """NaN in stale slots, unseen rows and the rows of others; NaN that is seen comes through."""
    C = _h()
    c = C.Case4([500, 300], 8, 2, 128, 16)
    plain = _decode(c, 100, 4, append, False)[0].clone()
    for b, n in enumerate(c.lens):
        for j in range(4, n - 100):
            c.blank(b, j)
    assert torch.equal(_decode(c, 100, 4, append, False)[0], plain)
    c.blank(0, 450)
    out = _decode(c, 100, 4, append, False)[0]
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[0]).all()) and torch.equal(out[1], plain[1])


def test_decode_bad_pages_and_lengths():
    C, gmc = _h(), _gmc()
    c = C.Case4([100, 100], 4, 2, 64, 16)
    good = _decode(c, 0, 0, True, False)[0].clone()
    c.table[1, 2] = -5
    out = _decode(c, 0, 0, True, False)[0]
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE and torch.equal(out[0], good[0])
    c.table[1, 6] = 1 << 20  # where the new row would go
    out = _decode(c, 0, 0, True, False)[0]
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE and torch.equal(out[0], good[0])


# ---- attend ------------------------------------------------------------------------------
ATTEND = [
    # lens, news, H, Hkv, d, page, window, sinks
    ([1], [1], 1, 1, 64, 16, 0, 0),
    ([24], [8], 4, 4, 128, 16, 0, 0),
    ([385, 300, 129, 128], [129, 44, 1, 128], 28, 4, 128, 16, 0, 0),
    ([385, 300, 5, 128], [129, 0, 5, 7], 8, 2, 64, 48, 0, 0),
    ([700], [300], 4, 4, 128, 256, 100, 4),
    ([700, 640], [257, 3], 4, 1, 64, 7, 64, 3),
    ([700], [2], 7, 1, 128, 64, 1, 0),
    ([200, 140], [90, 20], 2, 1, 256, 16, 70, 2),
    ([2000], [5], 4, 2, 128, 64, 0, 0),
    ([130, 0, 4], [2, 0, 6], 4, 2, 128, 16, 0, 0),  # more new tokens than tokens: queries before
    ([3000, 2999], [20, 1], 28, 4, 128, 64, 0, 0),   # two tiles, the key axis in parts
    ([1500], [40], 32, 32, 64, 16, 0, 0),
    ([900, 65], [3, 2], 100, 1, 128, 16, 200, 33),   # a tile a token
    ([700] * 6, [150] * 6, 14, 2, 128, 64, 0, 0),    # unpacked
    ([700] * 6, [150] * 6, 6, 2, 64, 48, 90, 7),
    ([1], [1], 1, 1, 256, 16, 0, 0),                 # 256 channels: token by token
    ([700, 0, 33, 5], [3, 0, 33, 9], 8, 2, 256, 48, 0, 0),
    ([900, 64], [40, 3], 11, 1, 256, 16, 100, 33),   # two launches
    ([257] * 8, [257] + [3] * 7, 2, 1, 256, 16, 0, 0),  # too many for that: unpacked
]


def _attend(c, window, sinks, **kw):
    cache = c.cache(max_len=min(max(c.lens) + 1, c.table.shape[1] * c.page))
    q = c.q.cuda()
    out = torch.full((len(q) + 1, c.H, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((len(q), c.H), 7.0, device="cuda")
    _gmc().attend(cache, q, out[:len(q)], max(c.news), q_offsets=c.offsets(), window=window,
                  sinks=sinks, lse=lse, **kw)
    return out, lse


@pytest.mark.parametrize("lens,news,H,Hkv,d,page,window,sinks", ATTEND)
def test_attend_matches_its_definition(lens, news, H, Hkv, d, page, window, sinks):
    from tests import cache_harness as A
    c = _h().Case4(lens, H, Hkv, d, page, news, spread=2.0)
    # what no query of a sequence sees may hold anything
    for b, (n, t) in enumerate(zip(lens, news)):
        if window:
            for j in range(sinks, n - t - window + 1):
                c.blank(b, j)
    out, lse = _attend(c, window, sinks)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    assert bool((out[-1] == 7.0).all())
    at = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        for x in range(t):
            ref, z, _, bound, size = A.attention(c.K[b], c.V[b], c.q[at + x], n - t + x, window,
                                                 sinks)
            _close(out[at + x], ref, bound, A.tolerance(c.dt, d, size, roundings=2),
                   f"sequence {b}, new token {x}")
            if n - t + x < 0:
                assert bool((lse[at + x] == -math.inf).all())
                continue
            _close(lse[at + x], z, torch.ones_like(z), A.lse_tolerance(d, size) * 4, "lse")
        at += t


@pytest.mark.parametrize("window,sinks", [(0, 0), (5000, 3), (100, 3)])
def test_attend_in_parts_that_fill_the_last_wave(window, sinks):
    """Unpacked, the key axis in parts although the tiles fill the GPU; some tokens of many."""
    from tests import cache_harness as A
    n, t = 8100, 2720
    c = _h().Case4([n], 8, 1, 64, 64, [t], spread=2.0)
    out, lse = _attend(c, window, sinks)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and bool((out[-1] == 7.0).all())
    for x in [0, 1, 15, 16, 127, 128, *range(201, t, 211), t - 2, t - 1]:
        ref, z, _, bound, size = A.attention(c.K[0], c.V[0], c.q[x], n - t + x, window, sinks)
        _close(out[x], ref, bound, A.tolerance(c.dt, 64, size, roundings=2), f"new token {x}")
        _close(lse[x], z, torch.ones_like(z), A.lse_tolerance(64, size) * 4, "lse")


@pytest.mark.parametrize("d,T", [(64, 5), (128, 5), (256, 5), (256, 33), (128, 200)])
def test_attend_with_and_without_offsets(d, T):
    """Strided queries and outputs, rows behind the last sequence, and as many tokens of each."""
    c = _h().Case4([400, 300, 350], 6, 2, d, 16, [T] * 3)
    want, z = _attend(c, 60, 2)
    q = torch.full((3 * T, 9, d + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    q[:, 1:7, :d] = c.q.cuda()
    out = torch.full((6, 3 * T + 2, d), 7.0, dtype=torch.bfloat16, device="cuda").permute(1, 0, 2)
    lse = torch.full((3 * T, 6), 7.0, device="cuda")
    cache = c.cache(max_len=min(401, c.table.shape[1] * c.page))
    _gmc().attend(cache, q[:, 1:7, :d], out[:3 * T], T, window=60, sinks=2, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and bool((out[3 * T:] == 7.0).all())
    assert torch.equal(out[:3 * T], want[:-1]) and torch.equal(lse, z)


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
def test_attend_of_one_token_a_sequence(window, sinks):
    """Without offsets it goes the way of decode."""
    from tests import cache_harness as A
    C, gmc = _h(), _gmc()
    c = C.Case4([500, 1, 0, 2000], 14, 2, 128, 64, spread=2.0)
    cache, q = c.cache(), c.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(4, 14, device="cuda")
    gmc.attend(cache, q, out, 1, window=window, sinks=sinks, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    for b, n in enumerate(c.lens):
        ref, z, _, bound, size = A.attention(c.K[b], c.V[b], c.q[b], n - 1, window, sinks)
        tol = C.tolerance(c, size)
        small = 2.0 ** -25 * c.V[b].double().abs().sum(0).repeat_interleave(7, 0)
        _close(out[b], ref, bound + small / tol, tol, f"sequence {b}")
        if n:
            _close(lse[b], z, torch.ones_like(z), A.lse_tolerance(128, size) * 4, "lse")
        else:
            assert bool((lse[b] == -math.inf).all())


@pytest.mark.parametrize("lens,news,H,Hkv", [([150, 200], [20, 7], 7, 1),
                                             ([700] * 6, [150] * 6, 14, 2)])
@pytest.mark.parametrize("which", ["k", "v", "both"])
def test_attend_does_not_see_what_it_should_not(lens, news, H, Hkv, which):
    """A key or value that is NaN reaches the rows that see it, and no others; both ways."""
    C = _h()
    c = C.Case4(lens, H, Hkv, 128, 16, news)
    plain, _ = _attend(c, 0, 0)
    bad = lens[0] - 4  # of the first sequence: its last four new tokens see it
    for pool, n in ((c.pool_k, "k"), (c.pool_v, "v")):
        if which in (n, "both"):
            for x in c.halves(pool):
                x[int(c.table[0, bad // c.page]), :, bad % c.page] = 0xf9
    out, _ = _attend(c, 0, 0)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    t = news[0]
    assert bool(torch.isnan(out[t - 4:t]).all())
    assert torch.isfinite(out[:t - 4]).all() and torch.equal(out[t:], plain[t:])
    # rows computed one by one: products in fp32, weights not rounded
    a, b = out[:t - 4].double(), plain[:t - 4].double()
    scale = float(b.abs().max())
    assert float((a - b).abs().max()) <= 2 * 2.0 ** -8 * scale


@pytest.mark.parametrize("news", [[3, 2], [300, 280]])
def test_attend_bad_pages_and_strides(news):
    C, gmc = _h(), _gmc()
    c = C.Case4([400, 300], 6, 2, 64, 16, news)
    good, _ = _attend(c, 0, 0)
    wide = torch.full((sum(news), 9, 72), math.nan, dtype=torch.bfloat16, device="cuda")
    q = wide[:, 1:7, :64]
    q.copy_(c.q)
    out = torch.full((6, sum(news), 64), 7.0, dtype=torch.bfloat16, device="cuda").permute(1, 0, 2)
    gmc.attend(c.cache(), q, out, max(news), q_offsets=c.offsets())
    torch.cuda.synchronize()
    assert torch.equal(out, good[:-1])
    c.table[1, 3] = -7
    out, _ = _attend(c, 0, 0)
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE and torch.equal(out[:news[0]], good[:news[0]])


def test_attend_equals_attend_of_the_unpacked_cache():
    """Unpacked to bf16 the cache gives the same bits: the values are exact."""
    from tests.cache_harness import Case
    C, gmc = _h(), _gmc()
    lens, news = [600, 333] * 4, [40, 333] * 4
    c = C.Case4(lens, 28, 4, 128, 64, news)
    out, lse = _attend(c, 0, 0)
    p = Case(lens, 28, 4, 128, "bf16", 128, news)
    p.K, p.V = c.K, c.V
    for b in range(8):
        p.put(b, range(p.lens[b]))
    cache = p.cache(max_len=601)
    want, z = torch.empty_like(out[:-1]), torch.empty_like(lse)
    gmc.attend(cache, c.q.cuda(), want, 333, q_offsets=c.offsets(), lse=z)
    torch.cuda.synchronize()
    assert torch.equal(out[:-1], want) and torch.equal(lse, z)


# ---- evict -------------------------------------------------------------------------------
@pytest.mark.parametrize("lens,Hkv,d,page,to_page,keep,sinks,recent", [
    ([1], 1, 64, 16, 16, 1, 0, 0), ([100, 7, 64], 2, 128, 16, 7, 30, 4, 10),
    ([1027, 300], 4, 128, 16, 16, 385, 4, 64), ([600], 1, 256, 48, 64, 123, 0, 1),
    ([500, 0, 33], 3, 64, 64, 16, 40, 1, 2)])
def test_evict_moves_the_packed_rows(lens, Hkv, d, page, to_page, keep, sinks, recent):
    C, gmc = _h(), _gmc()
    c = C.Case4(lens, Hkv, Hkv, d, page)
    cache = c.cache()
    to = C.Case4([keep] * c.B, Hkv, Hkv, d, to_page, seed=5, pad=16)
    dst = to.cache()
    dst.lens.zero_()
    scores = torch.rand(c.B, Hkv, max(lens), generator=c.gen)
    scores[:, :, ::5] = 0.25  # ties
    idx = torch.empty(c.B, Hkv, keep, dtype=torch.int32, device="cuda")
    kept = torch.empty(c.B, Hkv, keep, device="cuda")
    gmc.evict(cache, dst, scores.cuda(), keep, idx, kept, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    for b, n in enumerate(lens):
        m = min(keep, n)
        assert int(dst.lens[b]) == m
        for h in range(Hkv):
            rank = sorted(range(n), key=lambda j: (
                not (j < sinks or j >= n - recent), -float(scores[b, h, j]), j))
            want = sorted(rank[:m])
            assert idx[b, h, :m].tolist() == want and bool((idx[b, h, m:] == -1).all())
            if not m:
                continue
            for pool, dest in ((c.pool_k, to.dk), (c.pool_v, to.dv)):
                a, z = c.rows(pool, b, want), to.rows(dest.cpu(), b, range(m))
                assert torch.equal(a[0][:, h], z[0][:, h]) and torch.equal(a[1][:, h], z[1][:, h])
    # pages of nobody and the room behind a part stay
    assert bool((to.dk.cpu()[..., -16:] == 0xf9).all())


# ---- together ----------------------------------------------------------------------------
def test_calls_repeat_bit_for_bit_and_on_another_stream():
    C = _h()
    c = C.Case4([900, 411], 28, 4, 128, 64, [1, 1])
    a = _decode(c, 0, 0, True, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = _decode(c, 0, 0, True, True)
    torch.cuda.synchronize()
    for x, y in zip(a[:2] + a[3:], b[:2] + b[3:]):
        assert torch.equal(x, y)
