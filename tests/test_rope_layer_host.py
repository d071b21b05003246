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


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("batch", [True, False])
@pytest.mark.parametrize("layout", [BHND, BNHD])
def test_tensors_of_the_other_layout_are_refused(layout, batch, which):
    n = 2 if batch else 1
    p = layer(batch=n, text_tokens=0, qkv_layout=layout)
    r = rf2.RopePlan(heads=4, kv_heads=4, head_dim=64, axis_dims=(16, 24, 24))
    r.device = -1
    shape, other = ((n, 4, 192, 64), (n, 192, 4, 64)) if layout == BHND else ((n, 192, 4, 64), (n, 4, 192, 64))
    t = {x: torch.zeros((other if x == which else shape)[0 if batch else 1:], dtype=torch.bfloat16) for x in "qkv"}
    buf, w = p.alloc("cpu"), torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=f"^{which}: "):
        p.rf2_permute_rope(r, t["q"], t["k"], t["v"], torch.zeros(192, 3, dtype=torch.int32), buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], w, w,
                           stream=NoStream)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors are the host's, and with a device the call would be launched on them")
@pytest.mark.parametrize("shape", [(1, 192, 192, 64), (192, 192, 64), (192 * 192, 64), (-1,)], ids=str)
@pytest.mark.parametrize("layout", [BHND, BNHD])
def test_other_shapes_reach_the_device(layout, shape):
    # as many heads as tokens, views without heads
    p = rf2.Plan(batch=1, heads=192, head_dim=64, T=3, H=8, W=8, block=64, sparsity=0.5, qkv_layout=layout)
    r = rf2.RopePlan(heads=192, kv_heads=192, head_dim=64, axis_dims=(16, 24, 24))
    x, buf, w = torch.zeros(192 * 192 * 64, dtype=torch.bfloat16).view(shape), p.alloc("cpu"), torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(rf2.Rf2Error) as e:
        p.rf2_permute_rope(r, x, x, x, torch.zeros(192, 3, dtype=torch.int32), buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], w, w, stream=NoStream)
    assert e.value.code == rf2.RF2_ERR_HIP
