"""CPU tests of what the 4-bit cache, the rotated append and the read refuse (nothing launches)."""

import ctypes

import pytest
import torch

from tests.test_cache_args import (FAKE, _append, _attend, _attn, _cache, _decode, _evict, _rc,
                                   gmc)  # noqa: F401
from tests.test_cache_devices import OnDevice, Stream
from tests.test_cache_devices import gmc as launchless  # noqa: F401


def _cache4(gmc, **kw):  # noqa: F811
    part = 16 * 72
    f = dict(dtype=gmc.GMC_FP4, page_stride=4 * part, head_stride=part, slot_stride=0)
    f.update(kw)
    return _cache(gmc, **f)


def _rope(gmc, **kw):  # noqa: F811
    f = dict(table=FAKE, max_pos=100, rot=128, interleaved=0, sections=(0, 0, 0), H=28,
             q_row_stride=0, out_row_stride=0, new_row_stride=0)
    f.update(kw)
    f["sections"] = (ctypes.c_int * 3)(*f["sections"])
    return gmc.RopeStruct(**f)


def _turned(gmc, c, r, rows=6, T=3, pos=FAKE, k=FAKE, v=FAKE, q=FAKE, out=FAKE,  # noqa: F811
            off=None):
    return gmc.lib().gmc_cache_append_rope(ctypes.byref(c), ctypes.byref(r) if r else None, pos, k,
                                           v, q, out, off, rows, T, None)


def _read(gmc, c, rows=6, T=3, k=FAKE, v=FAKE, off=None):  # noqa: F811
    return gmc.lib().gmc_cache_read(ctypes.byref(c), k, v, off, rows, T, None)


BAD = [
    (dict(d=96), "UNSUPPORTED"), (dict(d=32), "UNSUPPORTED"), (dict(d=512), "UNSUPPORTED"),
    (dict(slot_stride=64), "ARG"), (dict(head_stride=16 * 72 - 16), "ARG"),
    (dict(head_stride=0), "ARG"), (dict(page_stride=16 * 71), "ARG"), (dict(page_stride=0), "ARG"),
    (dict(head_stride=16 * 72 + 8), "ARG"), (dict(page_stride=-16), "ARG"),
    (dict(k=FAKE + 8), "ARG"), (dict(v=None), "ARG"), (dict(max_len=129), "ARG"),
]


@pytest.mark.parametrize("change,code", BAD)
def test_every_operator_refuses_a_bad_4_bit_cache(gmc, change, code):  # noqa: F811
    c, want, a = _cache4(gmc, **change), _rc(gmc, code), _attn(gmc)
    assert _append(gmc, c) == want and _read(gmc, c) == want
    assert _turned(gmc, c, _rope(gmc, rot=min(128, c.d))) == want
    assert _attend(gmc, c, a) == want and _decode(gmc, c, a) == want
    good = _cache4(gmc, lens=FAKE + 256)
    assert _evict(gmc, c, good) == want and _evict(gmc, good, c) == want


def test_4_bit_caches_do_not_mix_with_others(gmc):  # noqa: F811
    c, to = _cache4(gmc), _cache(gmc, lens=FAKE + 256)
    assert _evict(gmc, c, to) == gmc.GMC_ERR_ARG
    assert _evict(gmc, _cache(gmc), _cache4(gmc, lens=FAKE + 256)) == gmc.GMC_ERR_ARG
    # and no other call takes the type
    pr = gmc.problem(1, 36, 36, 4, gmc.GMC_FP4)
    assert gmc.workspace_size(pr, 1296, 64, 28, 128, 3584, 257) == 0


def test_strides_of_a_single_head_or_page_are_anything(gmc):  # noqa: F811
    one = _cache4(gmc, Hkv=1, num_pages=1, head_stride=0, page_stride=0)
    assert _append(gmc, one, rows=0, off=FAKE) == gmc.GMC_OK
    assert _attend(gmc, _cache4(gmc), _attn(gmc, q_row_stride=4)) == gmc.GMC_ERR_ARG
    assert _attend(gmc, _cache4(gmc), _attn(gmc, q_row_stride=3588)) == gmc.GMC_ERR_ARG


def test_parts_of_pages_lie_apart(gmc):  # noqa: F811
    part, N = 16 * 72, _cache4(gmc).num_pages
    rows = lambda **kw: _read(gmc, _cache4(gmc, k=FAKE, **kw), rows=0, T=1,  # noqa: E731
                              off=FAKE)
    assert rows(page_stride=part, head_stride=N * part) == gmc.GMC_OK         # head after head
    assert rows(page_stride=9 * part, head_stride=2 * part) == gmc.GMC_OK     # with room between
    assert rows(page_stride=7 * part, head_stride=2 * part) == gmc.GMC_OK
    for page, head in ((1, 1), (3, 1), (2, 3), (6, 2), (1, N - 1), (2, 2 * N - 2), (4, 2)):
        assert rows(page_stride=page * part, head_stride=head * part) == gmc.GMC_ERR_ARG
    top = 1 << 62
    assert rows(page_stride=top, head_stride=top) == gmc.GMC_ERR_ARG
    assert rows(page_stride=16, head_stride=top) == gmc.GMC_ERR_ARG


def test_sizes(gmc):  # noqa: F811
    assert [gmc.cache4_part_size(p, d) for p, d in
            ((16, 128), (1, 64), (1, 128), (7, 64), (64, 256), (0, 64), (16, 96))] == \
        [1152, 48, 80, 256, 9216, 0, 0]
    bf16, c = _cache(gmc), _cache4(gmc)
    size = gmc.lib().gmc_attend_workspace_size
    # the unpacked rows: 2 sequences of one page of 128; 64 sequences of 32 pages
    wide = _cache4(gmc, d=256, page_stride=4 * 16 * 144, head_stride=16 * 144)
    assert size(ctypes.byref(wide), 28, 3) >= 2 * 128 * 4 * 256 * 4
    long = _cache4(gmc, B=64, max_pages=256)
    assert size(ctypes.byref(long), 28, 200) >= 64 * 4096 * 4 * 128 * 4
    # few tokens need none of it
    assert 0 < size(ctypes.byref(long), 28, 16) < 64 * 4096 * 4
    for cache in (wide, c, long):
        need, rows = size(ctypes.byref(cache), 28, 3), 3 * cache.B
        assert _attend(gmc, cache, _attn(gmc), rows=rows, n=need - 1) == gmc.GMC_ERR_WORKSPACE
    need = gmc.lib().gmc_decode_workspace_size(ctypes.byref(c), 28)
    assert need > 0 and _decode(gmc, c, _attn(gmc), n=need - 1) == gmc.GMC_ERR_WORKSPACE
    assert gmc.lib().gmc_evict_workspace_size(ctypes.byref(c), 4) == \
        gmc.lib().gmc_evict_workspace_size(ctypes.byref(bf16), 4)


@pytest.mark.parametrize("change,code", [
    (dict(table=None), "ARG"), (dict(table=FAKE + 8), "ARG"), (dict(max_pos=0), "ARG"),
    (dict(rot=0), "ARG"), (dict(rot=-16), "ARG"), (dict(rot=144), "ARG"),
    (dict(rot=24), "UNSUPPORTED"), (dict(rot=20), "UNSUPPORTED"), (dict(interleaved=2), "ARG"),
    (dict(sections=(16, 24, 23)), "ARG"), (dict(sections=(-1, 41, 24)), "ARG"),
    (dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 66)), "ARG"),
    (dict(H=30), "ARG"), (dict(H=-4), "ARG"), (dict(H=4 * 129), "UNSUPPORTED"),
    (dict(q_row_stride=28 * 128 - 8), "ARG"), (dict(q_row_stride=28 * 128 + 4), "ARG"),
    (dict(out_row_stride=128), "ARG"), (dict(out_row_stride=-8), "ARG"),
    (dict(new_row_stride=3 * 128), "ARG"), (dict(new_row_stride=4 * 128 + 2), "ARG")])
@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_rope_arguments(gmc, kind, change, code):  # noqa: F811
    c = _cache4(gmc) if kind == "fp4" else _cache(gmc)
    assert _turned(gmc, c, _rope(gmc, **change)) == _rc(gmc, code)


def test_rope_operands(gmc):  # noqa: F811
    c, r, E = _cache(gmc), _rope(gmc), gmc.GMC_ERR_ARG
    assert _turned(gmc, c, None) == E
    for k in ("k", "q", "out"):
        assert _turned(gmc, c, r, **{k: None}) == E
    for k in ("k", "v", "q", "out"):
        assert _turned(gmc, c, r, **{k: FAKE + 8}) == E
    assert _turned(gmc, c, r, pos=FAKE + 2) == E
    assert _turned(gmc, c, r, off=FAKE + 1) == E
    assert _turned(gmc, c, r, rows=5) == E and _turned(gmc, c, r, rows=-1, off=FAKE) == E
    assert _turned(gmc, c, r, T=0, rows=0) == E
    assert _turned(gmc, c, r, T=(1 << 30) + 1, rows=6, off=FAKE) == gmc.GMC_ERR_UNSUPPORTED
    assert _turned(gmc, c, _rope(gmc, H=0)) == E                            # queries of no head
    assert _turned(gmc, c, _rope(gmc, sections=(16, 24, 24)), pos=None) == E
    assert _turned(gmc, c, _rope(gmc, new_row_stride=4096), v=None) == E     # keys then values
    assert _turned(gmc, c, _rope(gmc, q_row_stride=8192)) == E              # in place, another stride
    assert _turned(gmc, _cache4(gmc), _rope(gmc, rot=48)) == gmc.GMC_ERR_UNSUPPORTED
    assert _turned(gmc, _cache(gmc, d=8, slot_stride=8), _rope(gmc, rot=16)) == E
    assert _turned(gmc, c, r, rows=0, off=FAKE, k=None, v=None, q=None, out=None) == gmc.GMC_OK


def test_read_operands(gmc):  # noqa: F811
    for c in (_cache(gmc), _cache4(gmc)):
        E = gmc.GMC_ERR_ARG
        assert _read(gmc, c, k=None) == E and _read(gmc, c, v=None) == E
        assert _read(gmc, c, k=FAKE + 8) == E and _read(gmc, c, v=FAKE + 4) == E
        assert _read(gmc, c, rows=7) == E and _read(gmc, c, off=FAKE + 2) == E
        assert _read(gmc, c, rows=0, off=FAKE, k=None, v=None) == gmc.GMC_OK


# ---- the binding -------------------------------------------------------------------------
B, HKV, H, PAGE, D = 2, 2, 4, 16, 64
PART = PAGE * D * 9 // 16


def _tensors(device=0, **at):
    f = dict(k=torch.zeros(4, HKV, PART, dtype=torch.uint8),
             v=torch.zeros(4, HKV, PART, dtype=torch.uint8),
             table=torch.zeros(B, 2, dtype=torch.int32), lens=torch.zeros(B, dtype=torch.int32),
             cos_sin=torch.zeros(50, D), q=torch.zeros(B, H, D, dtype=torch.bfloat16),
             out=torch.zeros(B, H, D, dtype=torch.bfloat16),
             k_new=torch.zeros(B, HKV, D, dtype=torch.bfloat16),
             v_new=torch.zeros(B, HKV, D, dtype=torch.bfloat16),
             pos=torch.zeros(B, dtype=torch.int32), offsets=torch.zeros(B + 1, dtype=torch.int32))
    f.update({n: t for n, t in at.items() if isinstance(t, torch.Tensor)})
    return {n: OnDevice(t, at.get(n) if isinstance(at.get(n), int) else device)
            for n, t in f.items()}


def _handles(g, o):
    g.library.gmc_cache4_part_size = lambda page, d: page * d * 9 // 16
    cache = g.KVCache4(o["k"], o["v"], o["table"], o["lens"], page_size=PAGE, d=D)
    return cache, g.Rope(o["cos_sin"])


def _call(g, o, stream=None, **kw):
    cache, rope = _handles(g, o)
    f = dict(positions=o["pos"], q=o["q"], out=o["out"], offsets=o["offsets"])
    f.update(kw)
    g.cache_append_rope(cache, rope, o["k_new"], o["v_new"], 1, stream=stream, **f)
    g.cache_read(cache, o["k_new"], o["v_new"], 1, offsets=f["offsets"], stream=stream)


def test_binding_passes_what_fits(launchless):  # noqa: F811
    _call(launchless, _tensors())
    _call(launchless, _tensors(), stream=Stream(0))
    assert launchless.library.calls == 4


@pytest.mark.parametrize("name", ["v", "table", "lens", "cos_sin", "q", "out", "k_new", "v_new",
                                  "pos", "offsets"])
@pytest.mark.parametrize("where", [-1, 1])
def test_binding_refuses_other_devices(launchless, name, where):  # noqa: F811
    with pytest.raises(launchless.GMCError):
        _call(launchless, _tensors(**{name: where}))
    assert launchless.library.calls == 0


@pytest.mark.parametrize("name,bad", [
    ("k", torch.zeros(4, HKV, PART)), ("k", torch.zeros(4, HKV, PART - 16, dtype=torch.uint8)),
    ("v", torch.zeros(4, HKV, PART + 16, dtype=torch.uint8)),
    ("cos_sin", torch.zeros(50, D, dtype=torch.float64)), ("cos_sin", torch.zeros(50, 63)),
    ("cos_sin", torch.zeros(D, 50).T), ("q", torch.zeros(B, H, D)),
    ("q", torch.zeros(B + 1, H, D, dtype=torch.bfloat16)),
    ("q", torch.zeros(B, D, H, dtype=torch.bfloat16).transpose(1, 2)),
    ("q", torch.zeros(1, H, D, dtype=torch.bfloat16).expand(B, H, D)),
    ("out", torch.zeros(B, H + 1, D, dtype=torch.bfloat16)),
    ("k_new", torch.zeros(B, HKV, D)), ("k_new", torch.zeros(B, HKV, 32, dtype=torch.bfloat16)),
    ("k_new", torch.zeros(B, 2 * HKV, D, dtype=torch.bfloat16)[:, ::2]),
    ("v_new", torch.zeros(B, 2 * HKV, D, dtype=torch.bfloat16)[:, HKV:]),  # another stride
    ("v_new", torch.zeros(B + 1, HKV, D, dtype=torch.bfloat16)),
    ("pos", torch.zeros(B, dtype=torch.int64)), ("pos", torch.zeros(3 * B, dtype=torch.int32)),
    ("offsets", torch.zeros(B, dtype=torch.int32))])
def test_binding_refuses_what_does_not_fit(launchless, name, bad):  # noqa: F811
    with pytest.raises(launchless.GMCError):
        _call(launchless, _tensors(**{name: bad}))
    assert launchless.library.calls == 0


def test_binding_refuses_odd_calls(launchless):  # noqa: F811
    g, o = launchless, _tensors()
    for kw in (dict(q=None), dict(out=None)):
        with pytest.raises(g.GMCError):
            _call(g, o, **kw)
    with pytest.raises(g.GMCError):
        _call(g, o, stream=Stream(1))
    cache, rope = _handles(g, o)
    for bad in ((1, 2), (1, 2, 3), (-1, 17, 16)):
        with pytest.raises(g.GMCError):
            g.Rope(o["cos_sin"], sections=bad)
    three = g.Rope(o["cos_sin"], sections=(8, 12, 12))
    with pytest.raises(g.GMCError):  # one position a row for three sections
        g.cache_append_rope(cache, three, o["k_new"], o["v_new"], 1, o["pos"])
    with pytest.raises(g.GMCError):  # the read's rows are dense
        g.cache_read(cache, OnDevice(torch.zeros(B, 2 * HKV, D, dtype=torch.bfloat16)[:, :HKV], 0),
                     o["v_new"], 1)
    assert g.library.calls == 0


def test_a_rope_keeps_few_layouts(launchless):  # noqa: F811
    """Every number of rows is a layout of its own."""
    g, o = launchless, _tensors()
    cache, rope = _handles(g, o)
    new = torch.zeros(3000, HKV, D, dtype=torch.bfloat16)
    for n in range(3000):
        g.cache_append_rope(cache, rope, OnDevice(new[:n], 0), OnDevice(new[:n], 0), 1,
                            offsets=o["offsets"])
    assert len(rope.layouts) <= 1024 and g.library.calls == 3000
