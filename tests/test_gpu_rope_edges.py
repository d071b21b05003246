"""Norms and rotations: calls of C that the binding does not make."""
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests.test_gpu_rope import Case

pytestmark = pytest.mark.gpu


def in_c(c, x):
    """An rf2_rows of a tensor of a case."""
    return c.plan._rows(x, "rows", x.shape)


@pytest.mark.parametrize("side", ["q", "k"])
@pytest.mark.parametrize("case", [dict(tokens=1, d=64, dims=(64,)), dict(), dict(tokens=300), dict(tokens=20000, heads=8, kv=8, d=64, dims=(16, 24, 24))], ids=str)
def test_gradients_of_weights_whose_side_is_left_out_are_sums_over_no_rows(case, side):
    # rows of one workgroup, of few, of enough for two launches of sums
    c = Case(**case)
    back, none = c.backward(), (0, 0, 0, 0)
    x, dz, w, at = (c.q, c.dq_out, c.wq, 0) if side == "q" else (c.k, c.dk_out, c.wk, 1)
    dx, dw = c.like(x), [torch.full((c.d,), float("nan"), device="cuda") for _ in range(2)]
    rows = [none] * 6
    rows[at::2] = [in_c(c, t) for t in (x, dz, dx)]
    pos, step = c.plan._pos(c.pos, *c.shape)
    weights = [w.data_ptr(), None] if side == "q" else [None, w.data_ptr()]
    ws = c.plan.alloc_workspace()
    code = rf2.lib().rf2_rope_backward(c.plan._h, *c.shape, rf2._two_rows_thrice.pack(*sum(rows, ())), pos, step, *weights, dw[0].data_ptr(), dw[1].data_ptr(),
                                       ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert code == rf2.RF2_OK
    assert torch.equal(dx, back[at]) and torch.equal(dw[at], back[2 + at])
    assert (dw[1 - at] == 0).all()
