"""CPU tests of the cache operators' argument checks (no compute call is made)."""

import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def gmc():
    from paper_2608_02134_gb300 import build
    build.build()
    from paper_2608_02134_gb300 import gmc as g
    g.lib()
    return g


FAKE = 1 << 20  # aligned, never dereferenced: the checks fail first


def _cache(gmc, **kw):
    f = dict(B=2, Hkv=4, d=128, dtype=gmc.GMC_BF16, page_size=16, num_pages=100, max_pages=8,
             max_len=0, page_stride=4 * 16 * 128, head_stride=16 * 128, slot_stride=128, k=FAKE,
             v=FAKE, page_table=FAKE, lens=FAKE, status=None)
    f.update(kw)
    return gmc.CacheStruct(**f)


BAD_CACHES = [
    (dict(B=0), "ARG"), (dict(Hkv=0), "ARG"), (dict(d=0), "ARG"), (dict(page_size=0), "ARG"),
    (dict(num_pages=0), "ARG"), (dict(max_pages=0), "ARG"), (dict(max_len=-1), "ARG"),
    (dict(max_len=129), "ARG"), (dict(dtype=9), "ARG"), (dict(k=None), "ARG"),
    (dict(v=None), "ARG"), (dict(page_table=None), "ARG"), (dict(lens=None), "ARG"),
    (dict(k=FAKE + 8), "ARG"), (dict(v=FAKE + 2), "ARG"), (dict(lens=FAKE + 1), "ARG"),
    (dict(status=FAKE + 2), "ARG"), (dict(slot_stride=132), "ARG"), (dict(head_stride=-8), "ARG"),
    (dict(page_stride=4), "ARG"), (dict(d=260), "UNSUPPORTED"), (dict(d=264), "UNSUPPORTED"),
    (dict(d=100), "UNSUPPORTED"), (dict(page_size=1 << 20, max_pages=1 << 12), "UNSUPPORTED"),
    (dict(B=70000), "UNSUPPORTED"),
]


def _rc(gmc, name):
    return {"ARG": gmc.GMC_ERR_ARG, "UNSUPPORTED": gmc.GMC_ERR_UNSUPPORTED,
            "WORKSPACE": gmc.GMC_ERR_WORKSPACE}[name]


def _attn(gmc, **kw):
    f = dict(H=28, window=0, sinks=0, scale=0.0)
    f.update(kw)
    return gmc.Attn(**f)


def _append(gmc, c, rows=6, T=3, k=FAKE, v=FAKE, off=None):
    return gmc.lib().gmc_cache_append(ctypes.byref(c), k, v, off, rows, T, None)


def _attend(gmc, c, a, rows=6, T=3, q=FAKE, out=FAKE, lse=None, off=None, ws=FAKE, n=1 << 40):
    return gmc.lib().gmc_attend(ctypes.byref(c), ctypes.byref(a) if a else None, q, off, rows, T,
                                out, lse, ws, n, None)


def _decode(gmc, c, a, q=FAKE, k=None, v=None, out=FAKE, lse=None, s=None, so=None, stride=128,
            ws=FAKE, n=1 << 40):
    return gmc.lib().gmc_decode(ctypes.byref(c), ctypes.byref(a) if a else None, q, k, v, out,
                                lse, s, so, stride, ws, n, None)


def _evict(gmc, c, to, s=FAKE, stride=128, keep=64, sinks=0, recent=0, idx=FAKE, os=None, ws=FAKE,
           n=1 << 40):
    return gmc.lib().gmc_evict(ctypes.byref(c), ctypes.byref(to), s, stride, keep, sinks, recent,
                               idx, os, ws, n, None)


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_every_operator_refuses_a_bad_cache(gmc, change, code):
    c, want = _cache(gmc, **change), _rc(gmc, code)
    a = _attn(gmc)
    assert _append(gmc, c) == want
    assert _attend(gmc, c, a) == want
    assert _decode(gmc, c, a) == want
    good = _cache(gmc, lens=FAKE + 256)
    assert _evict(gmc, c, good) == want
    assert _evict(gmc, good, c) == want


def test_null_cache(gmc):
    assert gmc.lib().gmc_cache_append(None, FAKE, FAKE, None, 6, 3, None) == gmc.GMC_ERR_ARG
    assert gmc.lib().gmc_attend_workspace_size(None, 28, 3) == 0


@pytest.mark.parametrize("change,code", [
    (dict(H=0), "ARG"), (dict(H=30), "ARG"), (dict(window=-1), "ARG"), (dict(sinks=-1), "ARG"),
    (dict(scale=-1.0), "ARG"), (dict(scale=float("nan")), "ARG"), (dict(scale=float("inf")), "ARG"),
    (dict(q_row_stride=4), "ARG"), (dict(q_head_stride=-8), "ARG"), (dict(out_row_stride=2), "ARG"),
    (dict(out_head_stride=12), "ARG"), (dict(H=4 * 129), "UNSUPPORTED")])
def test_attention_arguments(gmc, change, code):
    c, a = _cache(gmc), _attn(gmc, **change)
    assert _attend(gmc, c, a) == _rc(gmc, code)
    assert _decode(gmc, c, a) == _rc(gmc, code)


def test_attend_and_append_rows(gmc):
    c, a = _cache(gmc), _attn(gmc)
    E = gmc.GMC_ERR_ARG
    for f in (lambda **k: _append(gmc, c, **k), lambda **k: _attend(gmc, c, a, **k)):
        assert f(rows=5) == E            # B * T rows without offsets
        assert f(rows=-1, off=FAKE) == E
        assert f(T=0, rows=0) == E
        assert f(off=FAKE + 2) == E
    assert _append(gmc, c, k=None) == E
    assert _append(gmc, c, v=FAKE + 4) == E
    assert _attend(gmc, c, None) == E
    for k in ("q", "out", "ws"):
        assert _attend(gmc, c, a, **{k: None}) == E
        assert _attend(gmc, c, a, **{k: FAKE + 4}) == E
    assert _attend(gmc, c, a, lse=FAKE + 1) == E
    assert _attend(gmc, c, a, n=16) == gmc.GMC_ERR_WORKSPACE
    assert _append(gmc, c, rows=0, off=FAKE) == gmc.GMC_OK       # nothing to do
    assert _attend(gmc, c, a, rows=0, off=FAKE) == gmc.GMC_OK


def test_decode_arguments(gmc):
    c, a = _cache(gmc), _attn(gmc)
    E = gmc.GMC_ERR_ARG
    assert _decode(gmc, c, None) == E
    for k in ("q", "out", "ws"):
        assert _decode(gmc, c, a, **{k: None}) == E
        assert _decode(gmc, c, a, **{k: FAKE + 4}) == E
    assert _decode(gmc, c, a, k=FAKE) == E                        # keys without values
    assert _decode(gmc, c, a, v=FAKE) == E
    assert _decode(gmc, c, a, s=FAKE) == E                        # scores in without out
    assert _decode(gmc, c, a, so=FAKE) == E
    assert _decode(gmc, c, a, s=FAKE, so=FAKE, stride=127) == E   # fewer places than the cache
    assert _decode(gmc, c, a, n=16) == gmc.GMC_ERR_WORKSPACE


def test_evict_arguments(gmc):
    c, to = _cache(gmc), _cache(gmc, lens=FAKE + 256)
    E = gmc.GMC_ERR_ARG
    assert _evict(gmc, c, c) == E                                 # the same lengths
    for k in ("s", "idx", "ws"):
        assert _evict(gmc, c, to, **{k: None}) == E
        assert _evict(gmc, c, to, **{k: FAKE + 2}) == E
    assert _evict(gmc, c, to, keep=0) == E
    assert _evict(gmc, c, to, keep=129) == E                      # more than dst holds
    assert _evict(gmc, c, to, sinks=-1) == E
    assert _evict(gmc, c, to, recent=-1) == E
    assert _evict(gmc, c, to, sinks=40, recent=30) == E           # sinks + recent > keep
    assert _evict(gmc, c, to, stride=100) == E
    assert _evict(gmc, c, to, n=0) == gmc.GMC_ERR_WORKSPACE
    for change in (dict(B=3), dict(Hkv=2), dict(d=64), dict(dtype=gmc.GMC_F32)):
        assert _evict(gmc, c, _cache(gmc, lens=FAKE + 256, **change)) == E


def test_binding_refuses_tensors_that_do_not_fit(gmc):
    k = torch.zeros(4, 2, 16, 64)
    table, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(gmc.GMCError, match="device"):
        gmc.KVCache(k, k.clone(), table, lens)
    for bad in (dict(v=torch.zeros(4, 2, 16, 32)), dict(k=k.half(), v=k.half()),
                dict(k=k[..., ::2], v=k[..., ::2]), dict(table=table.long()),
                dict(lens=torch.zeros(2, dtype=torch.int32)), dict(lens=lens.long())):
        f = dict(k=k, v=k, table=table, lens=lens)
        f.update(bad)
        with pytest.raises(gmc.GMCError):
            gmc.KVCache(f["k"], f["v"], f["table"], f["lens"])
