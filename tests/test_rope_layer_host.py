"""The layer on raw projections, without a GPU: arguments of the binding that would be of no account."""
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests.test_rope_fused_host import layer

BHND, BNHD = rf2.RF2_LAYOUT_BHND, rf2.RF2_LAYOUT_BNHD


class NoStream:
    cuda_stream = 0


@pytest.mark.parametrize("over", [dict(pos=torch.zeros(192, 3, dtype=torch.int32)), dict(weights=(torch.ones(64), torch.ones(64))), dict(weights=(None, torch.ones(64)))],
                         ids=["pos", "weights", "one_weight"])
def test_positions_and_weights_without_a_plan_that_uses_them_are_refused(over):
    p = layer(text_tokens=0)
    x = torch.zeros(2, 4, 192, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="rope"):
        p.layer_fused(x, x, x, p.alloc("cpu"), stream=NoStream, **over)
