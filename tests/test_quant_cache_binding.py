"""What the binding of the calls over quantised caches refuses.  No GPU."""
import pytest
import torch

import paper_2508_17892_amd as il
from test_attention_binding import _cache, _device, _i32
from test_quant_cache_abi import _cache as _quant


def test_reading_in_a_type_that_is_not_the_rows():
    """A cache of the states' own type gives that type, tensors of the caller's have theirs: another one asked for was ignored without a word."""
    plain = _cache(_i32(1, 4), n_seq=1)
    with pytest.raises(TypeError, match="float32"):
        il.ilre_cache_read(plain, 2, dtype=torch.float32)
    for cache in (plain, _quant("fp8")):
        with pytest.raises(TypeError, match="float32"):
            il.ilre_cache_read(cache, 2, dtype=torch.float32, k_out=_device(2, 2, 128))
        with pytest.raises(TypeError, match="float32"):
            il.ilre_cache_read(cache, 0, dtype=torch.float32, v_out=_device(0, 2, 128))
        k = _device(0, 2, 128)
        assert il.ilre_cache_read(cache, 0, dtype=torch.bfloat16, k_out=k)[0] is k
        assert il.ilre_cache_read(cache, 0, k_out=k)[0] is k
