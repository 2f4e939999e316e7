"""The cache binding refuses tensors, streams and workspaces that are not on the cache's device,
and calls made while another device is the current one.  On the CPU, with tensors that say that
they lie on a device; the library is replaced, so that nothing can be launched."""

import pytest
import torch


class OnDevice:
    """A tensor that says that it lies on a device (-1: the host)."""

    def __init__(self, t, device):
        self.__dict__.update(t=t, device_=device)

    def __getattr__(self, name):
        return getattr(self.t, name)

    @property
    def is_cuda(self):
        return self.device_ >= 0

    def get_device(self):
        return self.device_


class Library:
    """Counts the calls that pass the checks."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        if name.endswith("_size"):
            return lambda *a: 256

        def call(*a):
            self.calls += 1
            return 0
        return call


class Stream:
    cuda_stream = 1234

    def __init__(self, device):
        self.device_index = device


@pytest.fixture
def gmc(monkeypatch):
    from paper_2608_02134_gb300 import gmc as g
    library = Library()
    monkeypatch.setattr(g, "lib", lambda: library)
    monkeypatch.setattr(g, "_current_device", lambda: 0)
    monkeypatch.setattr(g, "_current_stream", lambda device: 0)
    monkeypatch.setattr(g, "library", library, raising=False)
    return g


B, HKV, H, PAGE, D = 2, 2, 4, 16, 64


def _pools(device=0, **at):
    f = dict(k=torch.zeros(4, HKV, PAGE, D), v=torch.zeros(4, HKV, PAGE, D),
             page_table=torch.zeros(B, 2, dtype=torch.int32),
             lens=torch.zeros(B, dtype=torch.int32), status=torch.zeros(1, dtype=torch.int32))
    return {n: OnDevice(t, at.get(n, device)) for n, t in f.items()}


def _operands(device=0, **at):
    f = dict(q=torch.zeros(B, H, D), out=torch.zeros(B, H, D), lse=torch.zeros(B, H),
             k_new=torch.zeros(B, HKV, D), v_new=torch.zeros(B, HKV, D),
             scores=torch.zeros(B, HKV, 32), out_scores=torch.zeros(B, HKV, 32),
             offsets=torch.zeros(B + 1, dtype=torch.int32),
             out_idx=torch.zeros(B, HKV, 8, dtype=torch.int32), kept=torch.zeros(B, HKV, 8),
             workspace=torch.zeros(4096, dtype=torch.uint8))
    return {n: OnDevice(t, at.get(n, device)) for n, t in f.items()}


def _calls(gmc, o, cache, to, stream=None):
    """Every operator, with the names of the operands that it takes."""
    return {
        "append": (lambda: gmc.cache_append(cache, o["k_new"], o["v_new"], 1, offsets=o["offsets"],
                                            stream=stream), ("k_new", "v_new", "offsets")),
        "attend": (lambda: gmc.attend(cache, o["q"], o["out"], 1, q_offsets=o["offsets"],
                                      lse=o["lse"], workspace=o["workspace"], stream=stream),
                   ("q", "out", "offsets", "lse", "workspace")),
        "decode": (lambda: gmc.decode(cache, o["q"], o["out"], k_new=o["k_new"], v_new=o["v_new"],
                                      lse=o["lse"], scores=o["scores"],
                                      out_scores=o["out_scores"], workspace=o["workspace"],
                                      stream=stream),
                   ("q", "out", "k_new", "v_new", "lse", "scores", "out_scores", "workspace")),
        "evict": (lambda: gmc.evict(cache, to, o["scores"], 8, o["out_idx"], o["kept"],
                                    workspace=o["workspace"], stream=stream),
                  ("scores", "out_idx", "kept", "workspace")),
    }


OPERATORS = ["append", "attend", "decode", "evict"]


@pytest.mark.parametrize("op", OPERATORS)
def test_operands_on_the_caches_device_pass(gmc, op):
    cache, to = gmc.KVCache(**_pools()), gmc.KVCache(**_pools())
    _calls(gmc, _operands(), cache, to)[op][0]()
    _calls(gmc, _operands(), cache, to, Stream(0))[op][0]()
    assert gmc.library.calls == 2


@pytest.mark.parametrize("where", [-1, 1])
@pytest.mark.parametrize("name", ["k", "v", "page_table", "lens", "status"])
def test_every_tensor_of_a_cache_lies_on_one_device(gmc, name, where):
    with pytest.raises(gmc.GMCError, match="device"):
        gmc.KVCache(**_pools(**{name: where}))


def test_status_is_one_word(gmc):
    f = _pools()
    for bad in (torch.zeros(0, dtype=torch.int32), torch.zeros(1, dtype=torch.int64)):
        f["status"] = OnDevice(bad, 0)
        with pytest.raises(gmc.GMCError, match="status"):
            gmc.KVCache(**f)


@pytest.mark.parametrize("where", [-1, 1])
@pytest.mark.parametrize("op", OPERATORS)
def test_operands_elsewhere_are_refused(gmc, op, where):
    cache, to = gmc.KVCache(**_pools()), gmc.KVCache(**_pools())
    for name in _calls(gmc, _operands(), cache, to)[op][1]:
        call = _calls(gmc, _operands(**{name: where}), cache, to)[op][0]
        with pytest.raises(gmc.GMCError):
            call()
    assert gmc.library.calls == 0


def test_packed_rows_elsewhere_are_refused(gmc):
    cache = gmc.KVCache(**_pools())
    with pytest.raises(gmc.GMCError):
        gmc.cache_append(cache, OnDevice(torch.zeros(2 * B, HKV, D), 1), None, 1)
    assert gmc.library.calls == 0


@pytest.mark.parametrize("op", OPERATORS)
def test_another_current_device_is_refused(gmc, op, monkeypatch):
    cache, to = gmc.KVCache(**_pools()), gmc.KVCache(**_pools())
    monkeypatch.setattr(gmc, "_current_device", lambda: 1)
    with pytest.raises(gmc.GMCError, match="current device"):
        _calls(gmc, _operands(), cache, to)[op][0]()
    assert gmc.library.calls == 0


@pytest.mark.parametrize("op", OPERATORS)
def test_a_stream_of_another_device_is_refused(gmc, op):
    cache, to = gmc.KVCache(**_pools()), gmc.KVCache(**_pools())
    with pytest.raises(gmc.GMCError, match="stream"):
        _calls(gmc, _operands(), cache, to, Stream(1))[op][0]()
    assert gmc.library.calls == 0


def test_evict_to_a_cache_elsewhere_is_refused(gmc):
    cache, to = gmc.KVCache(**_pools()), gmc.KVCache(**_pools(device=1))
    with pytest.raises(gmc.GMCError, match="device"):
        _calls(gmc, _operands(), cache, to)["evict"][0]()
    assert gmc.library.calls == 0


@pytest.mark.parametrize("op", ["attend", "decode", "evict"])
def test_a_workspace_with_gaps_is_refused(gmc, op):
    # its count of elements would pass for as many bytes in a row
    cache, to = gmc.KVCache(**_pools()), gmc.KVCache(**_pools())
    o = _operands()
    o["workspace"] = OnDevice(torch.zeros(1, dtype=torch.uint8).expand(4096), 0)
    with pytest.raises(gmc.GMCError, match="workspace"):
        _calls(gmc, o, cache, to)[op][0]()
    assert gmc.library.calls == 0
