"""What the binding refuses before the library is called: host tensors that say they are on the device stand in for device tensors.  No GPU."""
import pytest
import torch

import paper_2508_17892_amd as il


class Device(torch.Tensor):
    is_cuda = property(lambda self: True)


def _device(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Device)


def _i32(*shape):
    return _device(*shape, dtype=torch.int32)


def _cache(table, n_seq=3):
    pages = _device(8, 2, 16, 128)
    return il.PagedKV(pages, pages, table, _i32(n_seq), _i32(n_seq + 1))


def test_a_page_table_expanded_over_sequences_is_refused():
    """Its row stride of 0 stands for contiguous rows in the C ABI, whose second row would lie behind the tensor."""
    with pytest.raises(ValueError):
        _cache(_i32(1, 4).expand(3, 4))
    # rows with something between them, and a lone row whatever its stride says
    assert _cache(_i32(3, 9)[:, 2:6]).c.table_stride == 9
    assert _cache(_i32(1, 4).expand(1, 4), n_seq=1).c.table_stride == 4
