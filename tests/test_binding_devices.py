"""Tensors on another device than the current one, whose stream the library works on, are refused.  No GPU: host tensors that say where they are stand in for device tensors."""
import pytest
import torch

import paper_2508_17892_amd as il
from test_attention_binding import Device, _cache, _device, _i32
from test_quant_cache_abi import _cache as _quant


class Elsewhere(Device):
    def get_device(self):
        return 1


@pytest.fixture(autouse=True)
def here(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)  # where host tensors are
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)


def _caches(name):
    cache = _cache(_i32(1, 4), n_seq=1) if name == "plain" else _quant("fp8")
    cache.k_pages = cache.k_pages.as_subclass(Device)
    return cache


@pytest.mark.parametrize("where", ["q", "out", "lse", "workspace", "cache"])
@pytest.mark.parametrize("kind", ["plain", "quantised"])
@pytest.mark.parametrize("call", ["paged", "tree"])
def test_attention(call, kind, where):
    cache = _caches(kind)
    t = dict(q=_device(2, 8, 128), out=_device(2, 8, 128), lse=_device(2, 8, dtype=torch.float32), workspace=_device(512, dtype=torch.uint8))
    if where == "cache":
        cache.k_pages = cache.k_pages.as_subclass(Elsewhere)
    else:
        t[where] = t[where].as_subclass(Elsewhere)
    q = t.pop("q")
    with pytest.raises(ValueError, match="device 1"):
        if call == "paged":
            il.ilre_paged_attention(q, cache, max_q=2, max_kv=64, **t)
        else:
            il.ilre_tree_attention(q, cache, _i32(2, 1), max_q=2, max_kv=64, **t)


@pytest.mark.parametrize("where", ["q", "k", "v", "q_out", "positions", "cache"])
@pytest.mark.parametrize("kind", ["plain", "quantised"])
@pytest.mark.parametrize("call", [il.ilre_rope_append, il.ilre_norm_rope_append])
def test_fill(call, kind, where):
    cache, freqs = _caches(kind), il.ilre_rope_frequencies(128, 10000.0)
    t = dict(q=_device(2, 8, 128), k=_device(2, 2, 128), v=_device(2, 2, 128), q_out=_device(2, 8, 128), positions=_i32(2))
    if where == "cache":
        cache.k_pages = cache.k_pages.as_subclass(Elsewhere)
    else:
        t[where] = t[where].as_subclass(Elsewhere)
    with pytest.raises(ValueError, match="device 1"):
        call(t["q"], t["k"], t["v"], cache, freqs, t["positions"], q_out=t["q_out"])
