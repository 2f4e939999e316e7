"""The key-value cache's operators on the GPU against their definitions in 64 bits."""

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


# ---- gmc_attend --------------------------------------------------------------------------
ATTEND = [
    # lens, news, H, Hkv, d, dtype, page, window, sinks
    ([1], [1], 1, 1, 64, "f32", 16, 0, 0),
    ([24], [8], 4, 4, 64, "f32", 16, 0, 0),
    ([130], [130], 4, 2, 128, "f32", 32, 0, 0),
    ([200, 3, 64, 65], [70, 3, 1, 64], 6, 2, 64, "f32", 16, 0, 0),
    ([300], [150], 4, 4, 128, "f32", 7, 33, 5),
    ([300], [40], 8, 1, 256, "f32", 16, 100, 1),
    ([97], [50], 5, 1, 36, "f32", 5, 0, 0),
    ([1], [1], 1, 1, 64, "bf16", 16, 0, 0),
    ([24], [8], 4, 4, 64, "bf16", 16, 0, 0),
    ([321], [64], 28, 4, 128, "bf16", 64, 0, 0),
    ([385, 300, 129, 128], [129, 44, 129, 1], 28, 4, 128, "bf16", 16, 0, 0),
    ([385, 300, 129, 128], [129, 44, 129, 1], 28, 4, 128, "bf16", 48, 0, 0),
    ([700], [700], 4, 2, 128, "bf16", 128, 0, 0),
    ([700], [700], 4, 2, 64, "bf16", 32, 0, 0),
    ([700], [300], 4, 4, 128, "bf16", 256, 100, 4),
    ([700], [700], 7, 1, 128, "bf16", 64, 1, 0),
    ([700], [700], 8, 8, 128, "bf16", 64, 128, 130),
    ([700], [257], 4, 1, 80, "bf16", 16, 64, 3),
    ([515], [200], 3, 1, 96, "bf16", 24, 50, 1),
    ([200], [90], 2, 1, 256, "bf16", 16, 70, 2),
    ([260], [60], 4, 2, 128, "bf16", 9, 0, 0),
    ([2000], [5], 4, 2, 128, "bf16", 64, 0, 0),
    ([2000], [3], 4, 2, 128, "f32", 64, 900, 17),
    ([150], [20], 40, 1, 128, "bf16", 16, 0, 0),
    ([90], [4], 100, 1, 64, "bf16", 16, 0, 0),
    ([130], [9], 128, 1, 64, "f32", 16, 40, 2),
]


def _attend(c, window=0, sinks=0, scale=None, max_len=None, strided=False, stream=None):
    gmc = _gmc()
    cache = c.cache(max_len=max_len)
    rows = sum(c.news)
    if strided:  # queries inside a wider projection, outputs head by head
        wide = torch.full((rows, c.H + 2, c.d + 8), math.nan, dtype=c.dt, device="cuda")
        q = wide[:, 1:c.H + 1, :c.d]
        q.copy_(c.q)
        out = torch.full((c.H, rows, c.d), 7.0, dtype=c.dt, device="cuda").permute(1, 0, 2)
    else:
        q = c.q.cuda()
        out = torch.full((rows, c.H, c.d), 7.0, dtype=c.dt, device="cuda")
    lse = torch.full((rows, c.H), 7.0, device="cuda")
    ragged = len(set(c.news)) > 1
    gmc.attend(cache, q, out, max(c.news), q_offsets=c.offsets() if ragged else None,
               window=window, sinks=sinks, scale=scale, lse=lse, stream=stream)
    return out, lse


def _check_attend(c, out, lse, window, sinks, scale=None):
    C = _harness()
    at = 0
    for b, (n, t) in enumerate(zip(c.lens, c.news)):
        for x in range(t):
            ref, z, _, bound, size = C.attention(c.K[b], c.V[b], c.q[at + x], n - t + x, window,
                                                 sinks, scale)
            tol = C.tolerance(c.dt, c.d, size, roundings=2)
            _close(out[at + x], ref, bound, tol, f"sequence {b}, new token {x}")
            _close(lse[at + x], z, torch.ones_like(z), C.lse_tolerance(c.d, size) * 4, "lse") \
                if n - t + x >= 0 else None
        at += t


@pytest.mark.parametrize("lens,news,H,Hkv,d,dtype,page,window,sinks", ATTEND)
def test_attend_matches_its_definition(lens, news, H, Hkv, d, dtype, page, window, sinks):
    c = _harness().Case(lens, H, Hkv, d, dtype, page, news, spread=2.0)
    out, lse = _attend(c, window, sinks)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, window, sinks)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_attend_strides_scale_and_slot_major_pools(dtype, d):
    c = _harness().Case([333, 70], 6, 2, d, dtype, 16, [50, 70], layout="slots")
    out, lse = _attend(c, 0, 0, scale=0.05, strided=True)
    torch.cuda.synchronize()
    _check_attend(c, out, lse, 0, 0, scale=0.05)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_rows_before_the_sequence_and_sequences_without_rows(dtype):
    # the second sequence holds fewer tokens than it has queries: the first queries see
    # nothing; the third has no queries, the fourth no tokens
    C = _harness()
    c = C.Case([40, 3, 9, 1], 4, 2, 128, dtype, 16, [5, 6, 0, 2])
    c.lens[3] = 0
    out, lse = _attend(c, max_len=48)
    torch.cuda.synchronize()
    _check_attend(_without_the_last(c), out, lse, 0, 0)
    assert torch.equal(out[5:8], torch.zeros_like(out[5:8]))
    assert bool((lse[5:8] == -math.inf).all())
    assert torch.equal(out[11:], torch.zeros_like(out[11:]))
    assert bool((lse[11:] == -math.inf).all())


def _without_the_last(c):
    """The case without its empty last sequence's keys."""
    c.K[3], c.V[3] = c.K[3][:0], c.V[3][:0]
    return c


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 128), ("f32", 16)])
def test_attend_values_that_are_not_seen_do_not_reach_a_row(dtype, page):
    # infinities and NaN in keys and values that only later queries, or none through the
    # window, may see
    C = _harness()
    c = C.Case([420], 4, 2, 128, dtype, page, [300])
    for j, x in ((30, math.nan), (260, math.inf), (310, math.nan), (419, -math.inf)):
        c.V[0][j, :, 5] = x
        c.put(0, [j])
    c.K[0][400] = math.nan
    c.put(0, [400])
    window, sinks = 40, 3
    out, _ = _attend(c, window, sinks)
    torch.cuda.synchronize()
    for x in range(300):
        i = 120 + x
        ok = C.seen(420, i, window, sinks)
        bad = [j for j in (30, 260, 310, 400, 419) if bool(ok[j])]
        if not bad:
            ref, _, _, bound, size = C.attention(c.K[0], c.V[0], c.q[x], i, window, sinks)
            _close(out[x], ref, bound, C.tolerance(c.dt, 128, size, roundings=2), f"query {x}")
        elif bad == [260] or bad == [310]:
            assert not bool(torch.isfinite(out[x, :, 5].float()).any())
            assert bool(torch.isfinite(out[x, :, 6].float()).all())


def test_attend_on_another_stream_twice_the_same():
    c = _harness().Case([600, 500], 28, 4, 128, "bf16", 64, [200, 100])
    side = torch.cuda.Stream()
    a, la = _attend(c)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b, lb = _attend(c, stream=side)
    side.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_marks_lengths_pages_and_offsets_out_of_range():
    gmc, C = _gmc(), _harness()
    c = C.Case([64, 64], 4, 2, 64, "bf16", 16, [4, 4])
    cache = c.cache()
    q, out = c.q.cuda(), torch.zeros(8, 4, 64, dtype=c.dt, device="cuda")

    def status(**kw):
        c.status.zero_()
        gmc.attend(cache, q, out, 4, **kw)
        torch.cuda.synchronize()
        return int(c.status.item())

    assert status() == 0
    c.dlens[0] = 65
    assert status() == gmc.STATUS_CACHE
    c.dlens[0] = -1
    assert status() == gmc.STATUS_CACHE
    c.dlens[0] = 64
    assert status(q_offsets=torch.tensor([0, 4, 9], dtype=torch.int32).cuda()) == gmc.STATUS_CACHE
    assert status(q_offsets=torch.tensor([4, 0, 4], dtype=torch.int32).cuda()) == gmc.STATUS_CACHE
    assert status() == 0
    cache.page_table[1, 2] = 1000
    assert status() == gmc.STATUS_CACHE
    cache.page_table[1, 2] = -7
    assert status() == gmc.STATUS_CACHE


# ---- gmc_decode --------------------------------------------------------------------------
DECODE = [
    # lens, H, Hkv, d, dtype, page, window, sinks
    ([1], 1, 1, 64, "f32", 16, 0, 0),
    ([1], 28, 4, 128, "bf16", 16, 0, 0),
    ([322], 28, 4, 128, "bf16", 16, 0, 0),
    ([17, 300, 16, 1, 129], 28, 4, 128, "bf16", 16, 0, 0),
    ([2085, 260], 28, 4, 128, "bf16", 64, 0, 0),
    ([2085, 260, 1100], 8, 8, 128, "bf16", 48, 128, 4),
    ([900, 33], 8, 1, 64, "bf16", 32, 1, 0),
    ([900, 33], 16, 1, 128, "bf16", 32, 500, 600),
    ([700], 40, 1, 128, "bf16", 16, 0, 0),
    ([500, 40], 4, 2, 256, "bf16", 16, 0, 0),
    ([500, 40], 4, 2, 80, "bf16", 7, 77, 3),
    ([5000], 2, 1, 128, "bf16", 128, 0, 0),
    ([333, 20], 4, 4, 64, "f32", 16, 0, 0),
    ([333, 20], 28, 4, 128, "f32", 16, 0, 0),
    ([1500, 7], 4, 2, 128, "f32", 64, 300, 2),
    ([600], 12, 4, 36, "f32", 5, 0, 0),
    ([300, 100], 6, 3, 256, "f32", 16, 0, 0),
    ([300, 100], 20, 1, 64, "f32", 16, 90, 9),
]


def _decode(c, window=0, sinks=0, scores=None, append=True, inplace=False, max_len=None):
    gmc = _gmc()
    new = None
    if append:
        new = [torch.stack([p[b][c.lens[b] - 1] for b in range(c.B)]).cuda() for p in (c.K, c.V)]
        for b in range(c.B):
            c.blank(b, c.lens[b] - 1)
    cache = c.cache(max_len=max_len)
    out = torch.full((c.B, c.H, c.d), 7.0, dtype=c.dt, device="cuda")
    lse = torch.full((c.B, c.H), 7.0, device="cuda")
    si = so = None
    if scores is not None:
        si = scores.cuda()
        so = si if inplace else torch.full_like(si, -5.0)
    gmc.decode(cache, c.q.cuda(), out, k_new=new and new[0], v_new=new and new[1], window=window,
               sinks=sinks, lse=lse, scores=si, out_scores=so)
    torch.cuda.synchronize()
    if append:  # the rows are in their pages, and nothing else changed
        for b in range(c.B):
            c.put(b, [c.lens[b] - 1])
        for dev, host in ((c.dk, c.pool_k), (c.dv, c.pool_v)):
            assert torch.equal(dev.cpu().view(torch.uint8), host.view(torch.uint8))
    return out, lse, so


@pytest.mark.parametrize("mode", ["plain", "scores", "inplace"])
@pytest.mark.parametrize("lens,H,Hkv,d,dtype,page,window,sinks", DECODE)
def test_decode_matches_its_definition(lens, H, Hkv, d, dtype, page, window, sinks, mode):
    C = _harness()
    c = C.Case(lens, H, Hkv, d, dtype, page, spread=2.0)
    S = max(lens) + 3
    scores = torch.rand(c.B, Hkv, S, generator=c.gen) if mode != "plain" else None
    out, lse, so = _decode(c, window, sinks, scores, inplace=mode == "inplace")
    assert int(c.status.item()) == 0
    for b, n in enumerate(lens):
        ref, z, w, bound, size = C.attention(c.K[b], c.V[b], c.q[b], n - 1, window, sinks)
        _close(out[b], ref, bound, C.tolerance(c.dt, d, size), f"sequence {b}")
        _close(lse[b], z, torch.ones_like(z), 4 * C.lse_tolerance(d, size), "lse")
        if scores is None:
            continue
        want = scores[b].double().clone()
        want[:, n - 1] = 0.0
        gain = w.reshape(Hkv, H // Hkv, n).sum(1)
        want[:, :n] += gain
        _close(so[b, :, :n], want[:, :n], gain + want[:, :n],
               4 * C.lse_tolerance(d, size), f"scores of {b}")
        hidden = ~C.seen(n, n - 1, window, sinks)
        assert torch.equal(so[b, :, :n].cpu()[:, hidden], scores[b, :, :n][:, hidden])
        rest = scores[b, :, n:] if mode == "inplace" else torch.full((Hkv, S - n), -5.0)
        assert torch.equal(so[b, :, n:].cpu(), rest)


def test_decode_of_a_cached_token_and_an_empty_sequence():
    C = _harness()
    c = C.Case([100, 1], 8, 2, 128, "bf16", 16)
    scores = torch.rand(2, 2, 100, generator=c.gen)
    c.lens[1] = 0
    out, lse, so = _decode(c, scores=scores, append=False, max_len=100)
    ref, z, w, bound, size = C.attention(c.K[0], c.V[0], c.q[0], 99)
    _close(out[0], ref, bound, C.tolerance(c.dt, 128, size), "out")
    want = scores[0].double() + w.reshape(2, 4, 100).sum(1)
    _close(so[0], want, want, 4 * C.lse_tolerance(128, size), "scores")
    assert torch.equal(out[1], torch.zeros_like(out[1]))
    assert bool((lse[1] == -math.inf).all())
    assert bool((so[1] == -5.0).all())


def test_decode_places_past_32_bit_offsets():
    # pools of more than 2^31 elements: the last pages' rows
    gmc, C = _gmc(), _harness()
    pages, page, Hkv, d = 5000, 1024, 4, 128
    k = torch.zeros(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    n = 1500
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    K, V = torch.randn(n, Hkv, d).bfloat16(), torch.randn(n, Hkv, d).bfloat16()
    for x in range(2):
        m = min(page, n - x * page)
        k[pages - 1 - x, :, :m] = K[x * page:x * page + m].permute(1, 0, 2).cuda()
        v[pages - 1 - x, :, :m] = V[x * page:x * page + m].permute(1, 0, 2).cuda()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    cache = gmc.KVCache(k, v, table, lens)
    q = torch.randn(1, 8, d).bfloat16()
    out = torch.empty(1, 8, d, dtype=torch.bfloat16, device="cuda")
    gmc.decode(cache, q.cuda(), out)
    ref, _, _, bound, size = C.attention(K, V, q[0], n - 1)
    _close(out[0], ref, bound, C.tolerance(torch.bfloat16, d, size), "out")
    out2 = torch.empty_like(out)
    gmc.attend(cache, q.cuda(), out2, 1)
    _close(out2[0], ref, bound, C.tolerance(torch.bfloat16, d, size, roundings=2), "attend")


# ---- gmc_evict ---------------------------------------------------------------------------
def _kept(scores, n, keep, sinks, recent):
    s = torch.where(torch.isnan(scores), torch.full_like(scores, -math.inf), scores).tolist()
    rank = sorted(range(n), key=lambda j: (not (j < sinks or j >= n - recent), -s[j], j))
    return sorted(rank[:min(keep, n)])


EVICT = [
    # lens, Hkv, d, dtype, page, to_page, keep, sinks, recent, scores
    ([1], 1, 64, "f32", 16, 16, 1, 0, 0, "rand"),
    ([20, 7], 2, 64, "bf16", 16, 16, 10, 2, 3, "rand"),
    ([500, 64, 10], 4, 128, "bf16", 16, 32, 64, 4, 16, "ties"),
    ([3000], 4, 128, "bf16", 64, 64, 1000, 4, 128, "rand"),
    ([3000], 2, 128, "f32", 48, 7, 999, 0, 0, "odd"),
    ([700, 699], 3, 80, "bf16", 5, 16, 350, 1, 349, "same"),
    ([9000], 1, 64, "bf16", 128, 16, 1, 1, 0, "rand"),
    ([40000], 1, 64, "bf16", 256, 256, 20001, 7, 100, "ties"),
    ([150000], 1, 8, "bf16", 256, 256, 333, 7, 100, "ties"),
    ([600] * 40, 8, 64, "bf16", 16, 16, 200, 4, 32, "rand"),
    ([64], 2, 64, "bf16", 16, 16, 16, 8, 8, "rand"),
]


@pytest.mark.parametrize("lens,Hkv,d,dtype,page,to_page,keep,sinks,recent,kind", EVICT)
def test_evict_matches_its_definition(lens, Hkv, d, dtype, page, to_page, keep, sinks, recent,
                                      kind):
    gmc, C = _gmc(), _harness()
    c = C.Case(lens, Hkv, Hkv, d, dtype, page)
    to = C.Case([keep] * c.B, Hkv, Hkv, d, dtype, to_page, seed=1)
    to.pool_k.fill_(math.nan)
    to.pool_v.fill_(math.nan)
    S = max(lens) + 5
    scores = torch.rand(c.B, Hkv, S, generator=c.gen)
    if kind == "ties":
        scores = (scores * 9).round() / 9 - 0.5
        scores[..., ::7] = -0.0
        scores[..., 3::11] = 0.0
    elif kind == "same":
        scores.fill_(0.25)
    elif kind == "odd":
        scores[..., 5] = math.nan
        scores[..., 9] = math.inf
        scores[..., 11:2500] = -math.inf
    src, dst = c.cache(), to.cache()
    to.dlens.fill_(-9)
    idx = torch.full((c.B, Hkv, keep), -7, dtype=torch.int32, device="cuda")
    kept = torch.full((c.B, Hkv, keep), -7.0, device="cuda")
    gmc.evict(src, dst, scores.cuda(), keep, idx, kept, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and int(to.status.item()) == 0
    assert to.dlens.tolist() == [min(keep, n) for n in lens]
    for b, n in enumerate(lens):
        m = min(keep, n)
        pages = to.table[b][torch.arange(m) // to_page].long()
        slots = torch.arange(m) % to_page
        for h in range(Hkv):
            want = _kept(scores[b, h], n, keep, sinks, recent)
            assert idx[b, h].tolist() == want + [-1] * (keep - m)
            same = kept[b, h, :m].cpu().view(torch.int32)
            assert torch.equal(same, scores[b, h, want].view(torch.int32))
            assert bool((kept[b, h, m:] == 0).all())
            to.pool_k[pages, h, slots] = c.K[b][want, h]
            to.pool_v[pages, h, slots] = c.V[b][want, h]
    for dev, host in ((to.dk, to.pool_k), (to.dv, to.pool_v)):
        assert torch.equal(dev.cpu().view(torch.uint8), host.view(torch.uint8))


# ---- gmc_cache_append --------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["heads", "slots"])
@pytest.mark.parametrize("lens,news,Hkv,d,dtype,page", [
    ([1], [1], 1, 64, "f32", 16), ([300, 40, 7], [300, 1, 3], 4, 128, "bf16", 16),
    ([1000], [513], 4, 128, "bf16", 48), ([90, 90], [33, 33], 2, 36, "f32", 7),
    ([64] * 9, [0, 1, 2, 3, 64, 5, 6, 7, 8], 3, 80, "bf16", 16)])
def test_append_puts_every_row_in_its_slot(lens, news, Hkv, d, dtype, page, layout):
    gmc, C = _gmc(), _harness()
    for packed in (False, True):
        c = C.Case(lens, Hkv, Hkv, d, dtype, page, news, layout=layout)
        for b, (n, t) in enumerate(zip(lens, news)):
            for j in range(n - t, n):
                c.blank(b, j)
        cache = c.cache()
        k = torch.cat([c.K[b][n - t:] for b, (n, t) in enumerate(zip(lens, news))])
        v = torch.cat([c.V[b][n - t:] for b, (n, t) in enumerate(zip(lens, news))])
        off = c.offsets() if len(set(news)) > 1 else None
        if packed:
            kv = torch.cat([p[b][n - t:] for b, (n, t) in enumerate(zip(lens, news))
                            for p in (c.K, c.V)])
            gmc.cache_append(cache, kv.cuda(), None, max(news), offsets=off)
        else:
            gmc.cache_append(cache, k.cuda(), v.cuda(), max(news), offsets=off)
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0
        for b, (n, t) in enumerate(zip(lens, news)):
            c.put(b, range(n - t, n))
        for dev, host in ((c.dk, c.pool_k), (c.dv, c.pool_v)):
            assert torch.equal(dev.cpu().view(torch.uint8), host.view(torch.uint8))


def test_append_drops_rows_before_the_sequence():
    gmc, C = _gmc(), _harness()
    c = C.Case([3], 2, 2, 64, "bf16", 16, [3])
    cache = c.cache()
    k = torch.randn(5, 2, 64).bfloat16()
    gmc.cache_append(cache, k.cuda(), k.cuda(), 5)
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE
    c.K[0], c.V[0] = k[2:], k[2:]
    c.put(0, range(3))
    assert torch.equal(c.dk.cpu().view(torch.uint8), c.pool_k.view(torch.uint8))
