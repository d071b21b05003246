"""Norms and rotations of Q and K without a GPU: the reference the kernels are tested against, configurations, arguments and refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests import rope_ref as ref

GOOD = dict(heads=4, kv_heads=2, head_dim=64, axis_dims=(16, 24, 24))


def make(**over):
    return rf2.RopePlan(**dict(GOOD, **over))


# ---- the reference ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("halves", [False, True])
def test_reference_rotates_pairs_by_their_angles(halves):
    rng = np.random.default_rng(1)
    pos = rng.integers(-50, 50, (3, 2))
    d, dims, theta = 16, (6, 8), 100.0
    x = rng.standard_normal((3, 2, d))
    z = ref.Rotation(pos, d, dims, theta, halves).turn(x)
    pair = 0
    for a, dim in enumerate(dims):
        for j in range(dim // 2):
            u, v = (pair, pair + d // 2) if halves else (2 * pair, 2 * pair + 1)
            for n in range(3):
                turned = (x[n, :, u] + 1j * x[n, :, v]) * np.exp(1j * pos[n, a] * theta ** (-2.0 * j / dim))
                assert np.allclose(z[n, :, u], turned.real, atol=1e-13) and np.allclose(z[n, :, v], turned.imag, atol=1e-13)
            pair += 1
    last = [(pair, pair + d // 2) if halves else (2 * pair, 2 * pair + 1)][0]
    assert np.array_equal(z[..., last], x[..., last])                   # a pair behind the last axis


def test_reference_depends_on_differences_of_positions_alone():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 64))
    dots = []
    for far in (0, 7, 123456789):
        at = [ref.Rotation(np.array([[p + far, 2 * far]]), 64, (40, 24)) for p in (3, 11)]
        dots.append((at[0].turn(q) * at[1].turn(k)).sum())
    assert np.allclose(dots, dots[0], rtol=0, atol=1e-9)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_reference_gradients_equal_differences(norm, halves):
    rng = np.random.default_rng(3)
    d, eps = 16, 1e-2
    rot = ref.Rotation(rng.integers(0, 100, (3, 2)), d, (6, 8), 50.0, halves)
    x, dz, w = rng.standard_normal((3, 2, d)), rng.standard_normal((3, 2, d)), 1 + 0.3 * rng.standard_normal(d)

    def loss(x, w):
        return (ref.forward(rot, x, w if norm else None, eps)[0] * dz).sum()

    dx, _, dw, _ = ref.backward(rot, x, dz, w if norm else None, eps)
    step = 1e-6
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = step
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - dx[i]) < 1e-7
    for i in range(d if norm else 0):
        e = np.zeros_like(w)
        e[i] = step
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * step) - dw[i]) < 1e-7


# ---- configurations ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bad", [dict(heads=0), dict(kv_heads=0), dict(heads=-1), dict(norm=2), dict(norm=-1), dict(eps=0.0), dict(eps=-1e-6), dict(eps=2.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(pairing=2), dict(pairing=-1), dict(axis_dims=(16, 23, 24)),
                                 dict(axis_dims=(-2, 24)), dict(axis_dims=(32, 34)), dict(axis_dims=(2 ** 31 - 2, 2 ** 31 - 2)),
                                 dict(axis_dims=(), norm=rf2.RF2_NORM_NONE), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")),
                                 dict(theta=float("inf")), dict(axis_dims=(4,), inv_freq=(1.0, float("nan"))), dict(axis_dims=(4,), inv_freq=(1.0, 1e6)),
                                 dict(axis_dims=(64,), theta=1e-9)], ids=str)
def test_invalid_configurations(bad):
    with pytest.raises(rf2.Rf2Error) as e:
        make(**bad)
    assert e.value.code == rf2.RF2_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(head_dim=256), dict(heads=65536), dict(kv_heads=65536)], ids=str)
def test_unsupported_configurations(bad):
    with pytest.raises(rf2.Rf2Error) as e:
        make(**bad)
    assert e.value.code == rf2.RF2_ERR_UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(dtype=torch.float32), dict(weight_dtype=torch.float64), dict(layout=2), dict(axis_dims=(2,) * 5),
                                 dict(axis_dims=(4,), inv_freq=(1.0,))], ids=str)
def test_arguments_that_the_binding_refuses(bad):
    with pytest.raises(ValueError):
        make(**bad)


def test_weights_of_the_other_type_are_refused():
    with pytest.raises(rf2.Rf2Error) as e:
        make(weight_dtype=torch.float16)
    assert e.value.code == rf2.RF2_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(), dict(axis_dims=()), dict(axis_dims=(64,)), dict(axis_dims=(0, 2, 0, 0)), dict(axis_dims=(16, 16, 16, 16)),
                                  dict(norm=rf2.RF2_NORM_NONE, eps=-1.0), dict(dtype=torch.float16, weight_dtype=torch.float32), dict(heads=65535, kv_heads=1),
                                  dict(theta=1e-3), dict(axis_dims=(4, 2), inv_freq=(0.5, -0.25, 0.0), theta=-1.0)], ids=str)
def test_sizes(over):
    p = make(**over)
    assert p.info.workspace_bytes == (0 if p.cfg.norm == rf2.RF2_NORM_NONE else 2 * (8192 * 64 * 4 + 128 * 64 * 8))
    assert p.alloc_workspace("cpu").numel() == p.info.workspace_bytes
    p.close()
    p.close()


# ---- arguments of the calls ----------------------------------------------------------------------------------------

AT = 0x10000


def tensors(names, **over):
    """rf2_rows of each name, dense [2, 5, 4 or 2 heads, 64]; `over` replaces (address, batch, token, head) of some."""
    rows = []
    for name in names:
        heads = 4 if "q" in name else 2
        rows += over.get(name, (AT, 5 * heads * 64, heads * 64, 64))
    return rf2.struct.pack("=" + "Qqqq" * len(names), *rows)


APPLY, BACKWARD = ("q", "k", "q_out", "k_out"), ("q", "k", "dq_out", "dk_out", "dq", "dk")


def apply_code(p, batch=2, tokens=5, pos=AT, pos_batch=0, wq=AT, wk=AT, **rows):
    return rf2.lib().rf2_rope_apply(p._h, batch, tokens, tensors(APPLY, **rows), pos, pos_batch, wq, wk, None)


def backward_code(p, batch=2, tokens=5, pos=AT, pos_batch=0, wq=AT, wk=AT, dwq=AT, dwk=AT, workspace=AT, **rows):
    return rf2.lib().rf2_rope_backward(p._h, batch, tokens, tensors(BACKWARD, **rows), pos, pos_batch, wq, wk, dwq, dwk, workspace, None)


needs_no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the calls that are in order would be launched on made-up addresses")
NONE = (0, 0, 0, 0)


def test_null_arguments():
    lib, bad = rf2.lib(), rf2.RF2_ERR_INVALID_ARG
    assert lib.rf2_rope_plan_create(None, None, None) == bad and lib.rf2_rope_plan_info(None, None) == bad
    assert lib.rf2_rope_plan_destroy(None) == rf2.RF2_OK
    assert lib.rf2_rope_apply(None, 1, 1, tensors(APPLY), None, 0, None, None, None) == bad
    assert lib.rf2_rope_backward(None, 1, 1, tensors(BACKWARD), None, 0, None, None, None, None, None, None) == bad
    p = make()
    assert lib.rf2_rope_apply(p._h, 1, 1, None, None, 0, None, None, None) == bad
    assert lib.rf2_rope_backward(p._h, 1, 1, None, None, 0, None, None, None, None, None, None) == bad


@needs_no_device
@pytest.mark.parametrize("over", [dict(), dict(batch=0), dict(tokens=0), dict(q=NONE, q_out=NONE, wq=None), dict(k=NONE, k_out=NONE, wk=None),
                                  dict(q=(AT, 0, 0, 0)), dict(q_out=(AT, 64, 2 * 64, 10 * 64)), dict(pos_batch=15),
                                  dict(batch=1, q_out=(AT, 0, 256, 64), k_out=(AT, 0, 128, 64)), dict(batch=1, tokens=1, q_out=(AT, 0, 0, 64), k_out=(AT, 0, 0, 64)),
                                  dict(q=(AT, 2 ** 40, 2 ** 32, 2 ** 50))], ids=str)
def test_calls_in_order_reach_the_device(over):
    assert apply_code(make(), **over) == rf2.RF2_ERR_HIP


@needs_no_device
@pytest.mark.parametrize("over", [
    dict(batch=-1), dict(tokens=-1), dict(pos_batch=-1), dict(pos_batch=2 ** 33), dict(pos=None), dict(pos=AT + 2), dict(wq=None), dict(wk=None), dict(wq=AT + 8),
    dict(wk=AT + 2), dict(q=NONE), dict(q_out=NONE), dict(k=NONE), dict(k_out=NONE), dict(q=NONE, q_out=NONE, k=NONE, k_out=NONE),
    dict(q=(AT + 8, 1280, 256, 64)), dict(k_out=(AT + 2, 640, 128, 64)), dict(q=(AT, 1280, 256, 60)), dict(k=(AT, 640, 132, 64)), dict(q=(AT, 1284, 256, 64)),
    dict(q=(AT, -1280, 256, 64)), dict(q=(AT, 1280, -256, 64)), dict(q=(AT, 1280, 256, -64)),
    # rows that are written and share memory
    dict(q_out=(AT, 1280, 256, 0)), dict(q_out=(AT, 0, 256, 64)), dict(q_out=(AT, 1280, 0, 64)), dict(q_out=(AT, 1280, 256, 56)), dict(q_out=(AT, 1280, 248, 64)),
    dict(q_out=(AT, 1272, 256, 64)), dict(k_out=(AT, 64, 64, 640)), dict(q_out=(AT, 2 ** 62, 256, 64)), dict(q=(AT, 2 ** 60, 256, 64)),
], ids=str)
def test_calls_that_are_refused(over):
    assert apply_code(make(), **over) == rf2.RF2_ERR_INVALID_ARG


@needs_no_device
def test_more_tokens_than_a_call_takes():
    p = make()
    rows = {n: (AT, 0, (4 if "q" in n else 2) * 64, 64) for n in APPLY}
    assert apply_code(p, batch=1, tokens=1 << 24, **rows) == rf2.RF2_ERR_HIP
    assert apply_code(p, batch=1, tokens=(1 << 24) + 1, **rows) == rf2.RF2_ERR_UNSUPPORTED
    assert apply_code(p, batch=2 ** 31 - 1, tokens=2 ** 31 - 1, **rows) == rf2.RF2_ERR_UNSUPPORTED


@needs_no_device
def test_no_norm_takes_no_weights_and_no_axes_no_positions():
    p = make(norm=rf2.RF2_NORM_NONE)
    assert apply_code(p, wq=None, wk=None) == rf2.RF2_ERR_HIP
    assert apply_code(p, wq=None) == rf2.RF2_ERR_INVALID_ARG and apply_code(p, wk=None) == rf2.RF2_ERR_INVALID_ARG
    assert apply_code(make(axis_dims=()), pos=None) == rf2.RF2_ERR_HIP


@needs_no_device
@pytest.mark.parametrize("over, code", [
    (dict(), "hip"), (dict(batch=0), "hip"), (dict(q=NONE, dq_out=NONE, dq=NONE, wq=None, dwq=None), "hip"), (dict(dq_out=(AT, 0, 0, 0)), "hip"),
    (dict(q=NONE), "bad"), (dict(dq=NONE), "bad"), (dict(dk_out=NONE), "bad"), (dict(dwq=None), "bad"), (dict(dwk=None), "bad"), (dict(dwq=AT + 2), "bad"),
    (dict(workspace=None), "bad"), (dict(workspace=AT + 8), "bad"), (dict(wq=None), "bad"), (dict(pos=None), "bad"), (dict(dq=(AT, 1280, 0, 64)), "bad"),
    (dict(dk=(AT, 640, 128, 32)), "bad"), (dict(dk_out=(AT, 640, 128, 4)), "bad"), (dict(tokens=-5), "bad"),
], ids=str)
def test_arguments_of_the_gradients(over, code):
    assert backward_code(make(), **over) == (rf2.RF2_ERR_HIP if code == "hip" else rf2.RF2_ERR_INVALID_ARG)


@needs_no_device
def test_gradients_without_a_norm_need_neither_rows_nor_workspace():
    p = make(norm=rf2.RF2_NORM_NONE)
    rest = dict(wq=None, wk=None, workspace=None)
    assert backward_code(p, q=NONE, k=NONE, dwq=None, dwk=None, **rest) == rf2.RF2_ERR_HIP
    assert backward_code(p, q=NONE, k=NONE, dwk=None, **rest) == rf2.RF2_ERR_INVALID_ARG


@pytest.mark.parametrize("change", ["dtype", "heads", "dim", "channels", "batch", "tokens", "pos", "pos type", "pos strides", "no weight", "weight", "weight type",
                                    "half a side", "nothing"])
def test_tensors_that_the_binding_refuses(change):
    p = make()
    p.device = -1                               # (the tensors here are the host's)
    t = dict(q=torch.zeros(2, 5, 4, 64), k=torch.zeros(2, 5, 2, 64), q_out=torch.zeros(2, 5, 4, 64), k_out=torch.zeros(2, 5, 2, 64))
    t = {n: x.bfloat16() for n, x in t.items()}
    t.update(pos=torch.zeros(5, 3, dtype=torch.int32), wq=torch.ones(64).bfloat16(), wk=torch.ones(64).bfloat16())
    t.update({"dtype": dict(q=t["q"].half()), "heads": dict(k=t["k"].repeat(1, 1, 2, 1)), "dim": dict(q_out=t["q_out"][..., :32]),
              "channels": dict(q=torch.zeros(2, 5, 64, 4).bfloat16().transpose(2, 3)), "batch": dict(k=t["k"][:1]), "tokens": dict(k_out=t["k_out"][:, :4]),
              "pos": dict(pos=t["pos"][:, :2].contiguous()), "pos type": dict(pos=t["pos"].long()), "pos strides": dict(pos=torch.zeros(3, 5).int().t()),
              "no weight": dict(wk=None), "weight": dict(wq=t["wq"][:32]), "weight type": dict(wq=t["wq"].float()), "half a side": dict(k_out=None),
              "nothing": dict(q=None, q_out=None, k=None, k_out=None)}[change])
    with pytest.raises(ValueError):
        p.rf2_rope_apply(t["q"], t["k"], t["pos"], t["q_out"], t["k_out"], t["wq"], t["wk"], stream=torch.cuda.default_stream() if torch.cuda.is_available() else NoStream)


class NoStream:
    cuda_stream = 0


def test_rows_of_the_binding_are_those_of_c():
    class rf2_rows(C.Structure):
        _fields_ = [("at", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]
    assert C.sizeof(rf2_rows * 4) == rf2._two_rows_twice.size and C.sizeof(rf2_rows * 6) == rf2._two_rows_thrice.size
    p = make(layout=rf2.RF2_LAYOUT_BHND)
    p.device = -1
    joint = torch.zeros(3, 7, 8, 64, dtype=torch.bfloat16)
    q = joint[:, :, 1:5].transpose(1, 2)
    assert p._sizes(q) == (3, 7, (3, 4, 7, 64), (3, 2, 7, 64)) and p._sizes(q[0]) == (1, 7, (4, 7, 64), (2, 7, 64))
    assert p._rows(q, "q", (3, 4, 7, 64)) == (joint.data_ptr() + 128, 7 * 512, 512, 64)
    assert p._rows(q[0], "q", (4, 7, 64)) == (joint.data_ptr() + 128, 0, 512, 64)
    p = make()
    p.device = -1
    q = joint[:, :, 1:5]
    assert p._sizes(q) == (3, 7, (3, 7, 4, 64), (3, 7, 2, 64)) and p._sizes(q[0]) == (1, 7, (7, 4, 64), (7, 2, 64))
    assert p._rows(q, "q", (3, 7, 4, 64)) == (joint.data_ptr() + 128, 7 * 512, 512, 64)
    assert p._rows(q[1], "q", (7, 4, 64)) == (joint.data_ptr() + 128 + 2 * 7 * 512, 0, 512, 64)
    assert math.isclose(p.cfg.theta, 10000.0)
