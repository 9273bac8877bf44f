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


@pytest.mark.parametrize("workspace", [torch.zeros(4096, dtype=torch.uint8), _device(16, dtype=torch.uint8).expand(4096, 16), _device(8192, dtype=torch.uint8)[::2]],
                         ids=["host", "expanded", "strided"])
def test_a_workspace_that_is_not_one_piece_of_device_memory_is_refused(workspace):
    """Its number of bytes says where the library may write, from its first one on."""
    cu = _i32(2)
    q, k = _device(2, 8, 128), _device(2, 2, 128)
    out, lse = _device(2, 8, 128), _device(2, 8, dtype=torch.float32)
    with pytest.raises(ValueError, match="workspace"):
        il.ilre_prompt_attention(q, k, k, cu, max_q=2, workspace=workspace, out=out, lse=lse)
    with pytest.raises(ValueError, match="workspace"):
        il.ilre_paged_attention(q, _cache(_i32(1, 4), n_seq=1), max_q=2, max_kv=64, workspace=workspace, out=out, lse=lse)
