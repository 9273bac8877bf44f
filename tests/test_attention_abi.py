"""Refusals of the operators around a recall: every bad argument is answered on the host, before any pointer is followed.  No GPU."""
import ctypes

import pytest
import torch

import paper_2508_17892_amd as il
from paper_2508_17892_amd import binding

FAKE = 1 << 20  # 256-byte aligned; never dereferenced: every call below fails validation first


def _opts(**kw):
    o = binding.IlreOpts()
    o.struct_size, o.dtype = ctypes.sizeof(binding.IlreOpts), il.ILRE_BF16
    for k, v in kw.items():
        setattr(o, k, v)
    return o


def _cache(**kw):
    c = il.IlrePagedKv()
    c.struct_size = ctypes.sizeof(il.IlrePagedKv)
    c.page_tokens, c.num_pages, c.Hkv, c.table_width, c.n_seq = 16, 10, 2, 4, 3
    c.k_pages = c.v_pages = c.page_table = c.kv_len = c.cu_q = FAKE
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _attn(**kw):
    a = il.IlreAttn(ctypes.sizeof(il.IlreAttn), 1, 0, 0, 1, 64, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _freqs(**kw):
    f = il.ilre_rope_frequencies(64, 10000.0)
    for k, v in kw.items():
        if k == "bad_freq":
            f.inv_freq[3] = v
        else:
            setattr(f, k, v)
    return f


def _ref(x):
    return None if x is None else ctypes.byref(x)


def paged(q=FAKE, out=FAKE, lse=FAKE, T=0, Hq=8, d=128, attn=_attn(), cache=None, strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_paged_attention(q, out, lse, T, Hq, d, _ref(attn), _ref(_cache() if cache is None else cache), _ref(strides), _ref(opts))


def prompt(q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=None, T=0, Tk=0, Hq=8, Hkv=2, d=128, cu_q=FAKE, cu_k=None, n_seq=1, attn=_attn(), strides=il.IlreStrides(),
           opts=_opts()):
    return il.load().ilre_prompt_attention(q, k, v, out, lse, T, Tk, Hq, Hkv, d, cu_q, cu_k, n_seq, _ref(attn), _ref(strides), _ref(opts))


def append(q=FAKE, q_out=FAKE, k=FAKE, v=FAKE, T=0, Hq=8, d=128, positions=None, freqs=_freqs(), pairing=0, cache=None, strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_rope_append(q, q_out, k, v, T, Hq, d, positions, _ref(freqs), pairing, _ref(_cache() if cache is None else cache), _ref(strides),
                                      _ref(opts))


def rope(x=FAKE, out=FAKE, T=0, H=8, d=128, positions=None, first=0, freqs=_freqs(), pairing=0, strides=il.IlreStrides(), opts=_opts()):
    return il.load().ilre_rope(x, out, T, H, d, positions, first, _ref(freqs), pairing, _ref(strides), _ref(opts))


def test_nothing_to_do_is_fine():
    assert paged() == prompt() == append() == rope() == il.ILRE_OK  # T = 0: validated, nothing launched
    assert append(q=None, q_out=None) == append(v=None, cache=_cache(v_pages=None)) == il.ILRE_OK


OPTS = [(dict(struct_size=8), il.ILRE_EINVAL), (dict(dtype=7), il.ILRE_EUNSUPPORTED), (dict(scale=-1.0), il.ILRE_EINVAL),
        (dict(scale=float("nan")), il.ILRE_EINVAL), (dict(flags=64), il.ILRE_EUNSUPPORTED), (dict(reserved=1), il.ILRE_EINVAL)]


@pytest.mark.parametrize("call", [paged, prompt, append, rope])
@pytest.mark.parametrize("kw,status", OPTS)
def test_opts(call, kw, status):
    assert call(opts=_opts(**kw)) == status
    assert il.ilre_last_error()


@pytest.mark.parametrize("call", [paged, prompt, append, rope])
def test_shapes_and_pointers_of_every_call(call):
    heads = "H" if call is rope else "Hq"
    assert call(opts=None) == call(strides=None) == il.ILRE_EINVAL
    assert call(T=-1) == call(**{heads: 0}) == il.ILRE_EINVAL
    assert call(d=64) == il.ILRE_EUNSUPPORTED
    assert call(T=1 << 30, **({"Tk": 1 << 30} if call is prompt else {})) == il.ILRE_EUNSUPPORTED
    assert call(T=1 << 25, **{heads: 2}, **({"Tk": 1 << 25} if call is prompt else {})) == il.ILRE_EUNSUPPORTED  # more than a launch has room for
    first = "x" if call is rope else "q"
    assert call(**{first: FAKE + 8}) == il.ILRE_EINVAL
    assert call(strides=il.IlreStrides(q_token=100)) == call(strides=il.IlreStrides(q_head=132)) == il.ILRE_EINVAL
    assert call(strides=il.IlreStrides(q_token=1 << 40)) == il.ILRE_EUNSUPPORTED
    assert call(strides=il.IlreStrides(out_token=12)) == il.ILRE_EINVAL


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(attn=None), dict(attn=_attn(struct_size=1)), dict(attn=_attn(causal=2)),
                                dict(attn=_attn(sink=-1)), dict(attn=_attn(window=-1)), dict(attn=_attn(causal=0, window=5)), dict(attn=_attn(sink=3)),
                                dict(attn=_attn(max_q=-1)), dict(attn=_attn(max_kv=-1)), dict(attn=_attn(total_kv=-1)), dict(lse=FAKE + 2),
                                dict(opts=_opts(workspace=FAKE + 8, workspace_bytes=1 << 20))])
def test_attention_arguments(kw):
    assert paged(**kw) == il.ILRE_EINVAL
    assert prompt(**kw) == il.ILRE_EINVAL


CACHE = [(dict(struct_size=0), 1), (dict(k_pages=None), 1), (dict(page_table=None), 1), (dict(kv_len=None), 1), (dict(cu_q=None), 1), (dict(n_seq=0), 1),
         (dict(num_pages=0), 1), (dict(table_width=0), 1), (dict(Hkv=0), 1), (dict(Hkv=3), 1), (dict(page_tokens=24), 1), (dict(page_tokens=0), 1),
         (dict(page_tokens=-16), 1), (dict(page_tokens=8), 2), (dict(page_tokens=65536), 2), (dict(k_pages=FAKE + 8), 1), (dict(v_pages=FAKE + 2), 1),
         (dict(stride_token=64, stride_head=2048, stride_page=4096), 1), (dict(stride_token=128, stride_head=2050, stride_page=4096), 1),
         (dict(stride_token=128, stride_head=0, stride_page=4096), 1), (dict(stride_token=1 << 40, stride_head=2048, stride_page=4096), 2),
         (dict(table_stride=3), 1)]


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_description(kw, status):
    assert paged(cache=_cache(**kw)) == status
    assert append(cache=_cache(**kw)) == status


def test_prompt_and_append_arguments():
    for kw in (dict(k=None, Tk=5, cu_k=FAKE), dict(v=None, Tk=5, cu_k=FAKE), dict(cu_q=None), dict(Hkv=0), dict(Hkv=3), dict(n_seq=0), dict(Tk=-1), dict(Tk=5), dict(k=FAKE + 4), dict(v=FAKE + 4),
               dict(strides=il.IlreStrides(k_token=64)), dict(strides=il.IlreStrides(v_head=130))):
        assert prompt(**kw) == il.ILRE_EINVAL, kw
    assert prompt(k=None, v=None) == il.ILRE_OK  # no keys at all
    assert prompt(Tk=5, cu_k=FAKE) == il.ILRE_OK and prompt(Tk=0x7FFFFFFF, cu_k=FAKE) == il.ILRE_EUNSUPPORTED
    for kw in (dict(k=None), dict(q=None), dict(q_out=None), dict(cache=_cache(v_pages=None)), dict(freqs=None), dict(freqs=_freqs(struct_size=3)),
               dict(freqs=_freqs(rotary=0)), dict(freqs=_freqs(rotary=144)), dict(freqs=_freqs(magnitude=float("inf"))), dict(freqs=_freqs(bad_freq=float("nan"))),
               dict(strides=il.IlreStrides(v_token=4)), dict(strides=il.IlreStrides(out_token=2048))):
        assert append(**kw) == il.ILRE_EINVAL, kw
    for kw in (dict(freqs=_freqs(rotary=24)), dict(pairing=2)):
        assert append(**kw) == rope(**kw) == il.ILRE_EUNSUPPORTED, kw
    assert rope(x=None) == rope(out=None) == rope(freqs=None) == rope(strides=il.IlreStrides(out_token=2048)) == il.ILRE_EINVAL
    assert rope(out=FAKE + 256, strides=il.IlreStrides(out_token=2048)) == il.ILRE_OK


def test_frequency_refusals():
    bad = [(dict(rotary=0), 1), (dict(rotary=130), 1), (dict(rotary=24), 2), (dict(base=0.0), 1), (dict(base=float("inf")), 1), (dict(scaling=9), 2),
           (dict(scaling=il.ILRE_ROPE_LINEAR, factor=0.5), 1), (dict(scaling=il.ILRE_ROPE_BANDS, factor=8.0), 1),
           (dict(scaling=il.ILRE_ROPE_BANDS, factor=8.0, low=4.0, high=4.0, original_len=100), 1),
           (dict(scaling=il.ILRE_ROPE_PARTS, factor=8.0, low=1.0, high=32.0, original_len=100, base=1.0), 1)]
    for kw, status in bad:
        kw = dict({"rotary": 64, "base": 10000.0}, **kw)
        with pytest.raises(il.IlreError) as e:
            il.ilre_rope_frequencies(kw.pop("rotary"), kw.pop("base"), **kw)
        assert e.value.status == status, kw


def test_workspace_sizing():
    def ws(T=1, n_seq=1, Hq=32, Hkv=8, d=128, max_q=1, max_kv=100000, total_kv=0, dtype=il.ILRE_BF16):
        return il.ilre_attention_workspace_bytes(T, n_seq, Hq, Hkv, d, max_q, max_kv, total_kv, dtype)
    assert ws(T=0) == 0 and ws(max_kv=16) == 0
    assert 0 < ws() < 64 << 20
    assert ws(T=16384, max_q=16384, max_kv=16384) == 0  # many rows need no ranges
    for kw, status in ((dict(T=-1), 1), (dict(n_seq=0), 1), (dict(Hkv=0), 1), (dict(Hq=30), 1), (dict(d=64), 2), (dict(dtype=5), 2), (dict(max_kv=-1), 1),
                       (dict(T=1 << 30), 2)):
        with pytest.raises(il.IlreError) as e:
            ws(**kw)
        assert e.value.status == status, kw


def test_binding_refuses_host_tensors_and_wrong_shapes():
    q, k = torch.zeros(2, 8, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        il.ilre_prompt_attention(q, k, k, torch.zeros(2, dtype=torch.int32), max_q=2)
    with pytest.raises(ValueError):
        il.ilre_rope(q, il.ilre_rope_frequencies(128, 10000.0))
    with pytest.raises(ValueError):
        il.PagedKV(torch.zeros(4, 2, 16, 128), None, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(il.IlreStrides) == 64
    assert ctypes.sizeof(il.IlrePagedKv) == 16 + 24 + 16 + 8 + 8 + 16 + 8
    assert il.IlrePagedKv.k_pages.offset == 40 and il.IlrePagedKv.table_width.offset == 88
    assert ctypes.sizeof(il.IlreAttn) == 32 and il.IlreAttn.total_kv.offset == 24
    assert ctypes.sizeof(il.IlreRopeFreqs) == 16 + 64 * 8
