"""GPU parity of quantised caches, head norms and reading back where calls are large or uneven: batches with one long context, chunks of a few thousand tokens, many heads, long reads."""
import pytest
import torch

import paper_2508_17892_amd as il
from test_gpu_attention import _announce
from test_gpu_quant_cache import Quant

pytestmark = pytest.mark.gpu


def uneven(long_at):
    """Lengths of 130 contexts."""
    return [9000 if i == long_at else 1 + 7 * i % 50 for i in range(130)]


@pytest.mark.parametrize("dtype,layout,long_at", [("bf16", "head", 0), ("bf16", "token", 129), ("f32", "head", 64)])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_one_long_context_among_many_short_ones(fmt, dtype, layout, long_at):
    """More lists than two for each compute unit, and one of them far longer than its share of the work."""
    _announce(f"quantised, one long context among 130 {fmt} {dtype} {layout}")
    x = Quant(fmt, [1] * 130, uneven(long_at), 8, 8, 64, dtype, layout, seed=long_at)
    out, lse = x.attend()
    torch.cuda.synchronize()
    x.check(out, lse)
    again, lse2 = x.attend()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    x.check(*x.attend(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")))
