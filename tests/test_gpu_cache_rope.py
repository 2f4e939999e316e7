"""Keys and queries turned by their positions on the way into the cache, against the rotation in
64 bits."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def _gmc():
    from paper_2608_02134_gb300 import gmc
    return gmc


def _table(n, rot, seed=0):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 1e4 ** (
        -torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
    return torch.cat([a.cos(), a.sin()], 1).float()


def _turn(x, table, pos, sections, interleaved):
    """Rows [t, heads, d] turned in 64 bits; pos [3, t] or [1, t].  Also sum of magnitudes."""
    rot = table.shape[1]
    n = rot // 2
    which = sum(([i] * m for i, m in enumerate(sections)), []) if sections else [0] * n
    c = torch.stack([table[pos[w], i] for i, w in enumerate(which)], 1).double()[:, None]
    s = torch.stack([table[pos[w], n + i] for i, w in enumerate(which)], 1).double()[:, None]
    x = x.double()
    y, size = x.clone(), x.abs()
    for i in range(n):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        a, b = x[..., p], x[..., q]
        y[..., p], y[..., q] = a * c[..., i] - b * s[..., i], b * c[..., i] + a * s[..., i]
        size[..., p] = size[..., q] = a.abs() + b.abs()
    return y, size


CASES = [
    # lens, news, H, Hkv, d, page, rot, interleaved, sections, dtype, layout
    ([1], [1], 1, 1, 64, 16, 64, False, None, "bf16", "plain"),
    ([5], [5], 2, 1, 16, 16, 16, False, None, "bf16", "plain"),
    ([5], [5], 2, 1, 16, 16, 16, True, None, "f32", "plain"),
    ([322], [1], 28, 4, 128, 16, 128, False, (16, 24, 24), "bf16", "packed"),
    ([40, 300, 7], [40, 130, 0], 28, 4, 128, 64, 128, False, (16, 24, 24), "bf16", "packed"),
    ([40, 300, 7], [3, 130, 7], 6, 2, 64, 48, 64, True, (5, 20, 7), "bf16", "apart"),
    ([40, 300, 7], [3, 130, 7], 6, 2, 96, 7, 32, False, (1, 2, 13), "f32", "packed"),
    ([90], [90], 8, 8, 80, 16, 80, False, None, "f32", "plain"),
    ([90, 33], [90, 33], 9, 3, 256, 16, 64, True, None, "bf16", "pair"),
    ([1], [1], 1, 1, 64, 16, 64, False, None, "fp4", "plain"),
    ([40, 300, 7], [40, 130, 0], 28, 4, 128, 64, 128, False, (16, 24, 24), "fp4", "packed"),
    ([40, 300, 7], [3, 130, 7], 6, 2, 64, 48, 32, True, (5, 4, 7), "fp4", "apart"),
    ([90, 33], [90, 33], 9, 3, 256, 16, 256, False, None, "fp4", "pair"),
    ([70], [64], 4, 2, 128, 16, 128, True, None, "fp4", "inplace"),
    ([70], [64], 4, 2, 128, 16, 96, False, None, "bf16", "inplace"),
    ([700], [650], 0, 2, 64, 16, 64, False, None, "bf16", "plain"),
]


# the places themselves as positions, too, where a row has one
@pytest.mark.parametrize("lens,news,H,Hkv,d,page,rot,interleaved,sections,dtype,layout,placed",
                         [c + (False,) for c in CASES] + [c + (True,) for c in CASES if not c[8]])
def test_rope_matches_its_definition(lens, news, H, Hkv, d, page, rot, interleaved, sections,
                                     dtype, layout, placed):
    from tests import cache4_harness as C4
    from tests import cache_harness as C
    gmc = _gmc()
    fp4 = dtype == "fp4"
    c = C4.Case4(lens, max(H, Hkv) // Hkv * Hkv, Hkv, d, page, news) if fp4 else \
        C.Case(lens, max(H, Hkv) // Hkv * Hkv, Hkv, d, dtype, page, news)
    for b in range(c.B):
        for j in range(lens[b] - news[b], lens[b]):
            c.blank(b, j)
    cache = c.cache()
    rows, g = sum(news), torch.Generator().manual_seed(11)
    raw = torch.randn(rows, H + 2 * Hkv, d, generator=g).to(c.dt)
    q, k, v = raw[:, :H], raw[:, H:H + Hkv], raw[:, H + Hkv:]
    most = 400
    if placed:
        pos = [torch.arange(n - t, n)[None] for n, t in zip(lens, news)]
    else:
        pos = [torch.randint(0, most, (3 if sections else 1, t), generator=g) for t in news]
    table = _table(max(most, max(lens)), rot)
    rope = gmc.Rope(table.cuda(), interleaved, sections)
    positions = None if placed else torch.cat([p.flatten() for p in pos]).int().cuda()
    wide = raw.cuda()
    out = torch.full((rows + 1, H, d), 7.0, dtype=c.dt, device="cuda")[:rows]
    if layout in ("packed", "inplace"):
        dq, dk, dv = wide[:, :H], wide[:, H:H + Hkv], wide[:, H + Hkv:]
        if layout == "inplace":
            out = dq
    elif layout == "apart":
        dq = q.cuda()
        kv = torch.full((rows, 2 * Hkv + 3, d), 9.0, dtype=c.dt, device="cuda")
        kv[:, 1:1 + Hkv], kv[:, 2 + Hkv:2 + 2 * Hkv] = k.cuda(), v.cuda()
        dk, dv = kv[:, 1:1 + Hkv], kv[:, 2 + Hkv:2 + 2 * Hkv]
        out = torch.full((rows, H + 5, d), 7.0, dtype=c.dt, device="cuda")[:, 2:2 + H]
    elif layout == "pair":  # as the compression's output lies
        dq, kv, at = q.cuda(), [], 0
        for t in news:
            kv += [k[at:at + t], v[at:at + t]]
            at += t
        dk, dv = torch.cat(kv).contiguous().cuda(), None
    else:
        dq, dk, dv = q.cuda(), k.contiguous().cuda(), v.contiguous().cuda()
    gmc.cache_append_rope(cache, rope, dk, dv, max(news), positions, dq if H else None,
                          out if H else None, offsets=c.offsets())
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    # a rounded product and sum in fp32, and the type's rounding
    tol = 3 * 2.0 ** -24 + (2.0 ** -8 if c.dt == torch.bfloat16 else 0.0)
    at = 0
    for b, (n, t) in enumerate(zip(lens, news)):
        if not t:
            continue
        if H:
            y, size = _turn(q[at:at + t], table, pos[b], sections, interleaved)
            got = out[at:at + t].cpu().double()
            assert bool(((got - y).abs() <= tol * size).all())
            assert torch.equal(got[..., rot:], y[..., rot:])
        y, size = _turn(k[at:at + t], table, pos[b], sections, interleaved)
        places = range(n - t, n)
        if fp4:
            C4.same_rows(c.rows(c.dk.cpu(), b, places),
                         C4.pack(y.float().bfloat16()), "keys")
            C4.same_rows(c.rows(c.dv.cpu(), b, places), C4.pack(v[at:at + t]), "values")
        else:
            p, j = c.table[b].long(), torch.arange(n - t, n)
            got = c.dk.cpu()[p[j // page], :, j % page].double()
            assert bool(((got - y).abs() <= tol * size).all())
            assert torch.equal(got[..., rot:], y[..., rot:])
            assert torch.equal(c.dv.cpu()[p[j // page], :, j % page], v[at:at + t])
        at += t
    if layout == "inplace":  # keys and values stay
        assert torch.equal(wide[:, H:].cpu(), raw[:, H:])
    # slots that are not new are as they were
    if not fp4:
        for b, (n, t) in enumerate(zip(lens, news)):
            p, j = c.table[b].long(), torch.arange(n - t)
            assert torch.equal(c.dk.cpu()[p[j // page], :, j % page], c.K[b][:n - t])


@pytest.mark.parametrize("dtype", ["bf16", "fp4"])
def test_rope_clamps_positions_and_drops_rows(dtype):
    """Positions outside the table, rows before the sequence and pages outside the pool are told
    and touch nothing they should not."""
    from tests import cache4_harness as C4
    from tests import cache_harness as C
    gmc = _gmc()
    c = C4.Case4([6], 2, 1, 64, 16) if dtype == "fp4" else C.Case([6], 2, 1, 64, "bf16", 16)
    cache = c.cache(max_len=16)
    table = _table(8, 64)
    rope = gmc.Rope(table.cuda())
    x = torch.randn(4, 1, 64).bfloat16()
    q = torch.randn(4, 2, 64).bfloat16()
    out = torch.empty_like(q).cuda()
    pos = torch.tensor([3, -2, 8, 2 ** 31 - 1], dtype=torch.int32)
    gmc.cache_append_rope(cache, rope, x.cuda(), x.cuda(), 4, pos.cuda(), q.cuda(), out)
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE
    y, size = _turn(q, table, pos[None].long().clamp(0, 7), None, False)
    assert bool(((out.cpu().double() - y).abs() <= (2.0 ** -8 + 2.0 ** -22) * size).all())
    # eight rows for a sequence of six
    c.status.zero_()
    x = torch.randn(8, 1, 64).bfloat16()
    pos = torch.zeros(8, dtype=torch.int32)
    gmc.cache_append_rope(cache, rope, x.cuda(), x.cuda(), 8, pos.cuda())
    k, v = (torch.empty(6, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert int(c.status.item()) == gmc.STATUS_CACHE
    gmc.cache_read(cache, k, v, 6)
    torch.cuda.synchronize()
    want = C4.unpack(*C4.pack(x[2:])) if dtype == "fp4" else x[2:].double()
    assert torch.equal(v.cpu().double(), want) and torch.equal(k.cpu().double(), want)
    # places as positions: the table ends before the sequence does
    c.status.zero_()
    cache.lens.fill_(12)
    gmc.cache_append_rope(cache, rope, x[:2].cuda(), x[:2].cuda(), 2)
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE
    c.table[0, 0] = -1
    cache = c.cache(max_len=16)
    before = c.dk.clone()
    gmc.cache_append_rope(cache, rope, x[:4].cuda(), x[:4].cuda(), 4, pos[:4].cuda())
    torch.cuda.synchronize()
    assert int(c.status.item()) == gmc.STATUS_CACHE
    assert torch.equal(c.dk.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_a_layer_step_through_one_graph(kind):
    """Turn, append, attend the prompt, then decode with scores, evict and decode on: the run
    of a layer, eager and its decode step captured and replayed."""
    from tests import cache4_harness as C4
    from tests import cache_harness as C
    gmc = _gmc()
    B, H, Hkv, d, page, T, room = 2, 14, 2, 128, 16, 50, 96
    g = torch.Generator().manual_seed(2)
    table = _table(room, d)
    rope = gmc.Rope(table.cuda())

    def empty(n):
        c = C4.Case4([room] * B, H, Hkv, d, page) if kind == "fp4" else \
            C.Case([room] * B, H, Hkv, d, "bf16", page)
        cache = c.cache(max_len=room)
        cache.lens.fill_(n)
        return c, cache

    c, cache = empty(T)
    prompt = torch.randn(B * T, H + 2 * Hkv, d, generator=g).bfloat16()
    x = prompt.cuda()
    q = torch.empty(B * T, H, d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    gmc.cache_append_rope(cache, rope, x[:, H:H + Hkv], x[:, H + Hkv:], T, q=x[:, :H], out=q)
    gmc.attend(cache, q, out, T)
    step = torch.zeros(B, H + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    tq = torch.empty(B, H, d, dtype=torch.bfloat16, device="cuda")
    token = torch.empty_like(tq)
    scores = torch.zeros(B, Hkv, room, device="cuda")
    ws = gmc.alloc_workspace(gmc.decode_workspace_size(cache, H))

    def one():
        cache.lens.add_(1)
        gmc.cache_append_rope(cache, rope, step[:, H:H + Hkv], step[:, H + Hkv:], 1, pos,
                              step[:, :H], tq)
        gmc.decode(cache, tq, token, scores=scores, out_scores=scores, workspace=ws)

    steps = torch.randn(6, B, H + 2 * Hkv, d, generator=g).bfloat16()
    graph = None
    rows, places = [prompt.reshape(B, T, -1, d)], list(range(T))
    for i in range(6):
        step.copy_(steps[i])
        pos.fill_(T + i)
        if i == 3:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one()
        if graph is not None:
            graph.replay()
        else:
            one()
        rows.append(steps[i][:, None])
        places.append(T + i)
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0
        all_rows = torch.cat(rows, 1)
        for b in range(B):
            p = torch.tensor(places)[None]
            k = _turn(all_rows[b, :, H:H + Hkv], table, p, None, False)[0].float().bfloat16()
            v = all_rows[b, :, H + Hkv:]
            qq = _turn(all_rows[b, -1:, :H], table, p[:, -1:], None, False)[0][0]
            if kind == "fp4":
                k, v = (C4.unpack(*C4.pack(z)).bfloat16() for z in (k, v))
            ref, _, _, bound, size = C.attention(k, v, tq[b].cpu(), T + i)
            assert bool(((tq[b].cpu().double() - qq).abs() <= 2.0 ** -7 * (qq.abs() + 1)).all())
            # a turned key may round the other way: one step more on a logit of `size`
            tol = 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -24 * (8 * d ** 0.5 * size + 64)
            off = (token[b].cpu().double() - ref).abs()
            if kind == "fp4":
                assert bool((off <= (tol + 2.0 ** -20) * bound).all())
            else:
                assert bool((off <= (tol + 2 * 2.0 ** -7 * size) * bound).all())
    total = scores.sum().item()
    assert abs(total - 6 * B * H) < 1e-3 * 6 * B * H
    to_c, to = empty(0)
    idx = torch.empty(B, Hkv, 40, dtype=torch.int32, device="cuda")
    kept = torch.empty(B, Hkv, 40, device="cuda")
    gmc.evict(cache, to, scores, 40, idx, kept, sinks=2, recent=5)
    ko, vo = (torch.empty(B * 40, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gmc.cache_read(to, ko, vo, 40)
    ka, va = (torch.empty(B * (T + 6), Hkv, d, dtype=torch.bfloat16, device="cuda")
              for _ in range(2))
    gmc.cache_read(cache, ka, va, T + 6)
    torch.cuda.synchronize()
    at = idx.long().permute(0, 2, 1)[..., None].expand(B, 40, Hkv, d)
    for got, src in ((ko, ka), (vo, va)):
        assert torch.equal(got.reshape(B, 40, Hkv, d),
                           src.reshape(B, T + 6, Hkv, d).gather(1, at))
