"""Norms and rotations: calls of C that the binding does not make, gradients that lie over the inputs, numbers that are not finite without a norm."""
import numpy as np
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests.test_gpu_rope import BHND, NONE, Case

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


@pytest.mark.parametrize("halves", [False, True])
def test_rotations_alone_of_rows_that_are_not_finite(halves):
    # the last pair does not turn, and token 0 is where no pair does
    c = Case(tokens=9, heads=2, kv=2, norm=NONE, halves=halves, dims=(44, 42, 40))
    c.pos[0] = 0
    c.rot = type(c.rot)(c.pos.cpu().numpy()[None], 128, (44, 42, 40), 10000.0, halves)
    want, _ = c.forward()
    partner = [(i + 64) % 128 if halves else i ^ 1 for i in range(128)]
    for n, i, value in [(n, i, value) for n in (0, 4) for i in (0, 5, 62, 63, 64, 127) for value in (float("inf"), float("-inf"), float("nan"))]:
        q, out = c.q.clone(), c.like(c.q)
        q[0, n, 1, i] = value
        c.plan.rf2_rope_apply(q, None, c.pos, out, None)
        pair = [i, partner[i]]
        got = out[0, n, 1, pair]
        assert not got.isfinite().any() and (not np.isnan(value) or got.isnan().all()), (n, i, value)
        out[0, n, 1, pair] = want[0, n, 1, pair]
        assert torch.equal(out, want), (n, i, value)


@pytest.mark.parametrize("case", [dict(), dict(layout=BHND), dict(joint=True, tokens=300, heads=16, kv=4), dict(joint=True, layout=BHND, batch=2, tokens=65),
                                  dict(halves=True, d=64, dims=(64,)), dict(tokens=3001, heads=40, kv=8, d=64, dims=(16, 24, 24))], ids=str)
def test_gradients_over_the_inputs(case):
    # dq over q and dk over k; with a joint projection its other columns stay
    c = Case(**case)
    want = c.backward()
    joint = case.get("joint")
    q, k = (c.q, c.k) if joint else (c.q.clone(), c.k.clone())
    v = (q.transpose(1, 2) if c.layout == BHND else q)._base if joint else None
    before = v.clone() if joint else None
    dw = [torch.full((c.d,), float("nan"), device="cuda") for _ in range(2)]
    c.plan.rf2_rope_backward(q, k, c.pos, c.dq_out, c.dk_out, q, k, c.wq, c.wk, *dw, c.plan.alloc_workspace())
    assert all(torch.equal(a, b) for a, b in zip(want, (q, k, *dw)))
    if joint:
        assert torch.equal(v[:, :, c.heads + c.kv:], before[:, :, c.heads + c.kv:])
