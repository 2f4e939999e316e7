"""The cache operators at shapes where their layouts change: many sequences, small and odd
head sizes, pages of every kind, rows of no sequence, other streams."""

import math

import pytest
import torch

from tests.test_gpu_cache import _attend, _check_attend, _close, _decode, _gmc, _harness, _kept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("d", [8, 16, 24, 40, 72, 104, 120])
def test_attend_small_and_odd_head_sizes(d):
    c = _harness().Case([150, 40], 6, 2, d, "bf16", 16, [60, 40], spread=2.0)
    out, lse = _attend(c, 30, 2)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, 30, 2)


@pytest.mark.parametrize("page", [8, 24, 40, 72, 136, 200, 384])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 5), (130, 150)])
def test_attend_pages_of_every_kind(page, window, sinks):
    c = _harness().Case([600, 137], 4, 2, 64, "bf16", page, [140, 70])
    out, lse = _attend(c, window, sinks)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, window, sinks)


@pytest.mark.parametrize("dtype,B", [("bf16", 40), ("bf16", 130), ("f32", 40)])
def test_attend_many_sequences(dtype, B):
    g = torch.Generator().manual_seed(B)
    news = torch.randint(0, 30, (B,), generator=g).tolist()
    lens = [t + int(torch.randint(0, 60, (1,), generator=g)) for t in news]
    lens = [max(1, n) for n in lens]
    c = _harness().Case(lens, 4, 2, 64, dtype, 16, news)
    out, lse = _attend(c, 20, 1)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out, lse, 20, 1)


@pytest.mark.parametrize("dtype,lens,news", [
    ("bf16", [3000], [5]), ("bf16", [300] * 6, [150, 1, 40, 0, 150, 2]), ("f32", [2000], [4])])
def test_attend_leaves_rows_of_no_sequence_alone(dtype, lens, news):
    gmc = _gmc()
    c = _harness().Case(lens, 4, 2, 64, dtype, 16, news)
    cache = c.cache()
    n = sum(news)
    q = torch.full((n + 9, 4, 64), math.nan, dtype=c.dt, device="cuda")
    q[2:2 + n] = c.q.cuda()
    out = torch.full_like(q, 7.0)
    lse = torch.full((n + 9, 4), 7.0, device="cuda")
    gmc.attend(cache, q, out, max(news), q_offsets=c.offsets() + 2, lse=lse)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    _check_attend(c, out[2:2 + n], lse[2:2 + n], 0, 0)
    for x in (out, lse):
        assert bool((x[:2] == 7.0).all()) and bool((x[2 + n:] == 7.0).all())


@pytest.mark.parametrize("B,H,Hkv,dtype,window,sinks", [
    (40, 8, 2, "bf16", 0, 0), (300, 4, 4, "bf16", 0, 0), (40, 4, 4, "f32", 17, 2),
    (70, 7, 1, "bf16", 20, 3), (33, 40, 1, "bf16", 0, 0)])
def test_decode_many_sequences_some_of_them_empty(B, H, Hkv, dtype, window, sinks):
    C = _harness()
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(1, 90, (B,), generator=g).tolist()
    c = C.Case(lens, H, Hkv, 64, dtype, 16)
    empty = [b for b in range(B) if b % 5 == 3]
    for b in empty:
        c.lens[b] = 0
    scores = torch.rand(B, Hkv, max(lens), generator=g)
    out, lse, so = _decode(c, window, sinks, scores, append=False, max_len=max(lens))
    assert int(c.status.item()) == 0
    for b in range(B):
        if b in empty:
            assert torch.equal(out[b], torch.zeros_like(out[b]))
            assert bool((lse[b] == -math.inf).all()) and bool((so[b] == -5.0).all())
            continue
        n = lens[b]
        ref, z, w, bound, size = C.attention(c.K[b], c.V[b], c.q[b], n - 1, window, sinks)
        _close(out[b], ref, bound, C.tolerance(c.dt, 64, size), f"sequence {b}")
        _close(lse[b], z, torch.ones_like(z), 4 * C.lse_tolerance(64, size), "lse")
        want = scores[b, :, :n].double() + w.reshape(Hkv, H // Hkv, n).sum(1)
        _close(so[b, :, :n], want, want, 4 * C.lse_tolerance(64, size), f"scores of {b}")


@pytest.mark.parametrize("dtype,H,Hkv,d", [("bf16", 28, 4, 128), ("f32", 8, 2, 64)])
def test_decode_strided_queries_and_slot_major_pools(dtype, H, Hkv, d):
    gmc, C = _gmc(), _harness()
    c = C.Case([700, 33], H, Hkv, d, dtype, 16, layout="slots")
    cache = c.cache()
    wide = torch.full((2, H + 3, d + 8), math.nan, dtype=c.dt, device="cuda")
    q = wide[:, 2:H + 2, :d]
    q.copy_(c.q)
    out = torch.full((H, 2, d), 7.0, dtype=c.dt, device="cuda").permute(1, 0, 2)
    gmc.decode(cache, q, out, scale=0.1)
    torch.cuda.synchronize()
    for b, n in enumerate(c.lens):
        ref, _, _, bound, size = C.attention(c.K[b], c.V[b], c.q[b], n - 1, scale=0.1)
        _close(out[b], ref, bound, C.tolerance(c.dt, d, size), f"sequence {b}")


def test_decode_marks_lengths_and_pages_out_of_range():
    gmc, C = _gmc(), _harness()
    c = C.Case([64, 64], 4, 2, 64, "bf16", 16)
    cache = c.cache()
    q, out = c.q.cuda(), torch.zeros(2, 4, 64, dtype=c.dt, device="cuda")

    def status():
        c.status.zero_()
        gmc.decode(cache, q, out)
        torch.cuda.synchronize()
        return int(c.status.item())

    assert status() == 0
    for bad in (65, -3):
        c.dlens[1] = bad
        assert status() == gmc.STATUS_CACHE
    c.dlens[1] = 64
    for bad in (1000, -7):
        cache.page_table[0, 1] = bad
        assert status() == gmc.STATUS_CACHE


def test_calls_on_another_stream_give_the_same():
    # everything that a call reads is made on the side stream just before it
    gmc, C = _gmc(), _harness()
    c = C.Case([900, 333], 8, 2, 128, "bf16", 16)
    scores = torch.rand(2, 2, 900, generator=c.gen)
    out, lse, so = _decode(c, scores=scores)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache = c.cache()
        q, s0 = c.q.cuda(), scores.cuda()
        o2, l2, s2 = torch.empty_like(out), torch.empty_like(lse), torch.full_like(s0, -5.0)
        new = [torch.stack([p[b][c.lens[b] - 1] for b in range(2)]).cuda() for p in (c.K, c.V)]
    gmc.decode(cache, q, o2, k_new=new[0], v_new=new[1], lse=l2, scores=s0, out_scores=s2,
               stream=side)
    to = C.Case([100, 100], 2, 2, 128, "bf16", 16, seed=4)
    with torch.cuda.stream(side):
        dst = to.cache()
        idx = torch.empty(2, 2, 100, dtype=torch.int32, device="cuda")
    gmc.evict(cache, dst, s2, 100, idx, recent=10, stream=side)
    side.synchronize()
    assert torch.equal(o2, out) and torch.equal(l2, lse) and torch.equal(s2, so)
    for b, n in enumerate(c.lens):
        for h in range(2):
            assert idx[b, h].tolist() == _kept(s2[b, h].cpu(), n, 100, 0, 10)


def test_calls_replayed_from_a_graph_give_the_same():
    gmc, C = _gmc(), _harness()
    c = C.Case([2500], 8, 2, 128, "bf16", 64, [40])
    cache = c.cache()
    q = c.q.cuda()
    out = torch.empty_like(q)
    ws = gmc.alloc_workspace(gmc.attend_workspace_size(cache, 8, 40))
    dq, dout = q[-1:].contiguous(), torch.empty_like(q[-1:])
    dws = gmc.alloc_workspace(gmc.decode_workspace_size(cache, 8))
    run = lambda: (gmc.attend(cache, q, out, 40, workspace=ws),          # noqa: E731
                   gmc.decode(cache, dq, dout, workspace=dws))
    run()
    torch.cuda.synchronize()
    want, dwant = out.clone(), dout.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        out.fill_(0)
        dout.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(dout, dwant)
