"""Refusals of the calls on quantised caches, head norms, axes and drafted trees: answered on the host, before any pointer is followed.  No GPU."""
import ctypes

import pytest
import torch

import paper_2508_17892_amd as il
import test_attention_abi as base
from test_attention_abi import FAKE, _attn, _freqs, _opts, _ref
from test_attention_binding import Device, _device, _i32

EINVAL, EUNSUPPORTED, OK = il.ILRE_EINVAL, il.ILRE_EUNSUPPORTED, il.ILRE_OK


def _quant(**kw):
    c = il.IlreQuantKv()
    c.kv = base._cache(struct_size=ctypes.sizeof(il.IlreQuantKv))
    c.format, c.k_scales, c.v_scales = il.ILRE_KV_FP8, FAKE, FAKE
    for k, v in kw.items():
        setattr(c if k in ("format", "reserved", "k_scales", "v_scales") else c.kv, k, v)
    return c


def _norms(**kw):
    n = il.IlreHeadNorms(ctypes.sizeof(il.IlreHeadNorms), 1, 1, 0.0, 1e-6, FAKE, FAKE)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _cache_ref(c):
    return None if c is None else ctypes.byref(c.kv if isinstance(c, il.IlreQuantKv) else c)


def _axes(*values):
    return (ctypes.c_uint8 * len(values))(*values)


def append(q=FAKE, q_out=FAKE, k=FAKE, v=FAKE, T=0, Hq=8, d=128, positions=None, n_axes=1, axes=None, freqs=_freqs(), pairing=0, norms=_norms(), cache=None,
           strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_norm_rope_append(q, q_out, k, v, T, Hq, d, positions, n_axes, axes, _ref(freqs), pairing, _ref(norms),
                                           _cache_ref(_quant() if cache is None else cache), _ref(strides), _ref(opts))


def turn(q=FAKE, out=FAKE, T=0, Hq=8, d=128, positions=None, n_axes=1, axes=None, freqs=_freqs(), pairing=0, norms=_norms(), strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_norm_rope(q, out, T, Hq, d, positions, n_axes, axes, 0, _ref(freqs), pairing, _ref(norms), _ref(strides), _ref(opts))


def read(k_out=FAKE, v_out=FAKE, T=0, d=128, tokens=None, cache=None, strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_cache_read(k_out, v_out, T, d, tokens, _cache_ref(_quant() if cache is None else cache), _ref(strides), _ref(opts))


def tree(q=FAKE, out=FAKE, lse=FAKE, T=0, Hq=8, d=128, tree=FAKE, words=1, stride=0, attn=_attn(causal=0), cache=None, strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_tree_attention(q, out, lse, T, Hq, d, tree, words, stride, _ref(attn), _cache_ref(_quant() if cache is None else cache), _ref(strides),
                                         _ref(opts))


def paged(cache, **kw):
    return il.load().ilre_paged_attention(FAKE, FAKE, FAKE, 0, 8, 128, _ref(_attn()), _cache_ref(cache), _ref(il.IlreStrides()), _ref(_opts(**kw)))


def test_nothing_to_do_is_fine():
    assert append() == turn() == read() == tree() == paged(_quant()) == OK  # T = 0: validated, nothing launched
    assert append(cache=base._cache()) == read(cache=base._cache()) == tree(cache=base._cache()) == OK
    assert append(q=None, q_out=None) == append(norms=None) == append(freqs=None) == turn(norms=None, freqs=None) == OK
    assert append(v=None, cache=_quant(v_pages=None, v_scales=None)) == read(v_out=None, cache=_quant(v_pages=None, v_scales=None)) == read(k_out=None) == OK
    assert append(norms=_norms(q_weight=None, k_weight=None)) == append(norms=_norms(q_norm=0, k_norm=0, eps=0.0, offset=1.0)) == OK
    assert append(cache=_quant(format=il.ILRE_KV_FP4, stride_token=256, stride_head=128, stride_page=4096)) == OK
    assert append(positions=FAKE, n_axes=3, axes=_axes(*[j % 3 for j in range(32)])) == OK


@pytest.mark.parametrize("call", [append, turn, read, tree])
@pytest.mark.parametrize("kw,status", base.OPTS)
def test_opts(call, kw, status):
    assert call(opts=_opts(**kw)) == status
    assert il.ilre_last_error()


@pytest.mark.parametrize("call", [append, turn, read, tree])
def test_shapes_and_strides_of_every_call(call):
    assert call(opts=None) == call(strides=None) == call(T=-1) == EINVAL
    assert call(d=64) == call(T=1 << 30) == EUNSUPPORTED
    token, head = ("k_token", "k_head") if call is read else ("q_token", "q_head")
    assert call(strides=il.IlreStrides(**{token: 100})) == call(strides=il.IlreStrides(**{head: 132})) == EINVAL
    assert call(strides=il.IlreStrides(**{token: 1 << 40})) == EUNSUPPORTED
    assert call(**{"k_out" if call is read else "q": FAKE + 8}) == EINVAL


QUANT = [(dict(struct_size=100), EINVAL), (dict(format=0), EUNSUPPORTED), (dict(format=3), EUNSUPPORTED), (dict(reserved=1), EINVAL), (dict(k_scales=None), EINVAL),
         (dict(v_scales=None), EINVAL), (dict(k_scales=FAKE + 2), EINVAL), (dict(v_scales=FAKE + 1), EINVAL),
         (dict(stride_token=144, stride_head=4096, stride_page=8192), EINVAL), (dict(stride_token=128, stride_head=2080, stride_page=8192), EINVAL),
         (dict(stride_token=128, stride_head=2048, stride_page=8224), EINVAL)]


@pytest.mark.parametrize("kw,status", QUANT + [(k, s) for k, s in base.CACHE if "struct_size" not in k])
def test_cache_description(kw, status):
    assert append(cache=_quant(**kw)) == read(cache=_quant(**kw)) == paged(_quant(**kw)) == status or kw == dict(Hkv=3) and read(cache=_quant(**kw)) == OK
    assert tree(cache=_quant(**kw)) == status
    old = il.load().ilre_rope_append(FAKE, FAKE, FAKE, FAKE, 0, 8, 128, None, _ref(_freqs()), 0, _cache_ref(_quant(**kw)), _ref(il.IlreStrides()), _ref(_opts()))
    assert old == status


def test_norms_axes_and_positions():
    for kw in (dict(norms=_norms(struct_size=8)), dict(norms=_norms(q_norm=2)), dict(norms=_norms(k_norm=-1)), dict(norms=_norms(eps=-1e-6)), dict(norms=_norms(eps=float("nan"))), dict(norms=_norms(eps=1e-40)), dict(norms=_norms(eps=1e39)),
               dict(norms=_norms(eps=float("inf"))), dict(norms=_norms(offset=float("inf"))), dict(norms=_norms(q_weight=FAKE + 8)), dict(norms=_norms(k_weight=FAKE + 2)),
               dict(n_axes=0), dict(n_axes=-1), dict(n_axes=3), dict(n_axes=3, positions=FAKE), dict(n_axes=3, axes=_axes(*[0] * 32)),
               dict(n_axes=3, positions=FAKE, axes=_axes(*[0] * 31, 3)), dict(axes=_axes(1, *[0] * 31)), dict(positions=FAKE + 2),
               dict(freqs=_freqs(struct_size=3)), dict(freqs=_freqs(rotary=0)), dict(strides=il.IlreStrides(out_token=2048))):
        assert append(**kw) == turn(**kw) == EINVAL, kw
    for kw in (dict(n_axes=9, positions=FAKE, axes=_axes(*[0] * 32)), dict(pairing=2), dict(freqs=_freqs(rotary=24))):
        assert append(**kw) == turn(**kw) == EUNSUPPORTED, kw
    for kw in (dict(k=None), dict(q=None), dict(q_out=None), dict(cache=_quant(v_pages=None)), dict(strides=il.IlreStrides(k_token=64))):
        assert append(**kw) == EINVAL, kw
    assert turn(q=None) == turn(out=None) == EINVAL
    assert il.load().ilre_rope_append(FAKE, FAKE, FAKE, FAKE, 0, 8, 128, None, None, 0, _cache_ref(_quant()), _ref(il.IlreStrides()), _ref(_opts())) == EINVAL


def test_read_and_tree_arguments():
    for kw in (dict(k_out=None, v_out=None), dict(tokens=FAKE + 1), dict(cache=_quant(v_pages=None)), dict(cache=_quant(Hkv=0)), dict(strides=il.IlreStrides(v_head=4))):
        assert read(**kw) == EINVAL, kw
    assert il.load().ilre_cache_read(FAKE, FAKE, 0, 128, None, None, _ref(il.IlreStrides()), _ref(_opts())) == EINVAL
    for kw in (dict(tree=None), dict(tree=FAKE + 2), dict(words=0), dict(words=-1), dict(words=2, stride=1), dict(stride=-1), dict(attn=_attn()), dict(attn=_attn(causal=1, window=4)),
               dict(attn=_attn(causal=0, max_q=33)), dict(q=None), dict(out=None), dict(lse=FAKE + 2)):
        assert tree(**kw) == EINVAL, kw
    assert tree(attn=_attn(causal=0, max_q=33), words=2) == tree(words=1, stride=5) == OK


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(il.IlreQuantKv) == 96 + 8 + 16 and il.IlreQuantKv.k_scales.offset == 104
    assert ctypes.sizeof(il.IlreHeadNorms) == 40 and il.IlreHeadNorms.eps.offset == 16 and il.IlreHeadNorms.k_weight.offset == 32


# ------------------------------------------------------------------------------------------------ the binding

def _codes(fmt, *shape):
    return torch.zeros(*shape, 128 if fmt == "fp8" else 64, dtype=torch.uint8).view(torch.float8_e4m3fn if fmt == "fp8" else torch.uint8).as_subclass(Device)


def _cache(fmt, codes=None, scales=None, **kw):
    codes = _codes(fmt, 8, 2, 16) if codes is None else codes
    scales = _device(8, 2, 16, 4, dtype=torch.uint8) if scales is None else scales
    args = dict(dict(v_pages=codes, v_scales=scales), **kw)
    return il.QuantKV(codes, args["v_pages"], scales, args["v_scales"], _i32(3, 4), _i32(3), _i32(4))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_quantised_caches_of_the_binding(fmt):
    c = _cache(fmt).quant
    assert (c.kv.stride_page, c.kv.stride_head, c.kv.stride_token, c.format) == (4096, 2048, 128, 1 if fmt == "fp8" else 2)
    assert c.kv.struct_size == ctypes.sizeof(il.IlreQuantKv)
    token = lambda t: t.permute(0, 2, 1, 3)  # noqa: E731
    c = _cache(fmt, token(_codes(fmt, 8, 16, 2)), token(_device(8, 16, 2, 4, dtype=torch.uint8))).quant
    assert (c.kv.stride_page, c.kv.stride_head, c.kv.stride_token) == (4096, 128, 256)
    # keys and values of a page side by side
    both, scales = _codes(fmt, 8, 2, 2, 16), _device(8, 2, 2, 16, 4, dtype=torch.uint8)
    c = _cache(fmt, both[:, 0], scales[:, 0], v_pages=both[:, 1], v_scales=scales[:, 1]).quant
    assert (c.kv.stride_page, c.kv.stride_head) == (8192, 2048) and c.kv.v_pages - c.kv.k_pages == (4096 if fmt == "fp8" else 2048) and c.v_scales - c.k_scales == 128
    assert _cache(fmt, v_pages=None, v_scales=None).v_pages is None
    with pytest.raises(ValueError, match="layout"):
        _cache(fmt, token(_codes(fmt, 8, 16, 2)))
    with pytest.raises(ValueError):
        _cache(fmt, scales=_device(8, 2, 16, 8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        _cache(fmt, scales=_device(8, 2, 16, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        _cache(fmt, v_scales=None)
    with pytest.raises(ValueError, match="expanded"):
        _cache(fmt, _codes(fmt, 1, 2, 16).expand(8, 2, 16, -1), _device(1, 2, 16, 4, dtype=torch.uint8).expand(8, 2, 16, 4))
    with pytest.raises(TypeError):
        il.QuantKV(_device(8, 2, 16, 128), None, _device(8, 2, 16, 4, dtype=torch.uint8), None, _i32(3, 4), _i32(3), _i32(4))
    with pytest.raises(il.IlreError):
        _cache(fmt, _codes(fmt, 8, 2, 16)[..., :32])


def test_arguments_of_the_binding():
    cache, freqs = _cache("fp8"), il.ilre_rope_frequencies(64, 10000.0)
    q, k = _device(2, 8, 128), _device(2, 2, 128)
    f32 = _device(2, 2, 128, dtype=torch.float32)
    weight = _device(128)
    for bad in (_device(127), _device(2, 128), _device(256)[::2], torch.zeros(128)):
        with pytest.raises(ValueError):
            il.HeadNorms(bad)
    with pytest.raises(TypeError):
        il.HeadNorms(weight, _device(128, dtype=torch.float32))
    for kw, error in ((dict(norms=il.HeadNorms(_device(128, dtype=torch.float32))), TypeError), (dict(axes=(0,) * 31, positions=_i32(1, 2)), ValueError),
                      (dict(axes=(0,) * 32, positions=_i32(2)), ValueError), (dict(axes=(0,) * 32), ValueError), (dict(axes=(0,) * 32, positions=_i32(1, 3)), ValueError),
                      (dict(axes=(0,) * 32, positions=_i32(2, 4)[:, ::2]), ValueError), (dict(axes=(300,) * 32, positions=_i32(1, 2)), ValueError),
                      (dict(positions=_i32(3)), ValueError), (dict(q_out=_device(2, 7, 128)), ValueError)):
        with pytest.raises(error):
            il.ilre_norm_rope_append(q, k, k, cache, freqs, **dict(dict(q_out=_device(2, 8, 128)), **kw))
    with pytest.raises(TypeError):
        il.ilre_norm_rope_append(q, f32, f32, cache, freqs, q_out=q)
    with pytest.raises(ValueError):
        il.ilre_norm_rope_append(q, k, k, _cache("fp8", v_pages=None, v_scales=None), freqs, q_out=q)
    for kw in (dict(k_out=_device(3, 2, 128)), dict(k_out=_device(2, 3, 128)), dict(k_out=k, v_out=f32), dict(k_out=k, tokens=_i32(3)), dict(k_out=torch.zeros(2, 2, 128))):
        with pytest.raises(ValueError):
            il.ilre_cache_read(cache, 2, **kw)
    with pytest.raises(ValueError):
        il.ilre_cache_read(_cache("fp8", v_pages=None, v_scales=None), 2, v_out=k)
    out, lse, ws = _device(2, 8, 128), _device(2, 8, dtype=torch.float32), _device(512, dtype=torch.uint8)
    for bad in (_i32(3, 1), _i32(2), _device(2, 1, dtype=torch.int64), torch.zeros(2, 1, dtype=torch.int32), _i32(2, 4)[:, ::2], _i32(1, 1).expand(2, 1)):
        with pytest.raises(ValueError, match="tree"):
            il.ilre_tree_attention(q, cache, bad, max_q=2, max_kv=64, workspace=ws, out=out, lse=lse)
    with pytest.raises(ValueError, match="workspace"):
        il.ilre_tree_attention(q, cache, _i32(2, 1), max_q=2, max_kv=64, workspace=torch.zeros(512, dtype=torch.uint8), out=out, lse=lse)
