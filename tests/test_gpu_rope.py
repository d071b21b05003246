"""Rows of Q and K normalised and rotated, and the gradients, against the formulas in 64 bits; tolerances in tests/rope_ref.py."""
import numpy as np
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests import rope_ref as ref

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NONE, RMS, BHND, BNHD = rf2.RF2_NORM_NONE, rf2.RF2_NORM_RMS, rf2.RF2_LAYOUT_BHND, rf2.RF2_LAYOUT_BNHD


def f64(t):
    return t.detach().cpu().double().numpy()


class Case:
    """Inputs on the device, as a program has them, and as [batch, tokens, heads, d] in 64 bits."""

    def __init__(self, *, batch=1, tokens=37, heads=4, kv=2, d=128, dims=(44, 42, 42), theta=10000.0, halves=False, norm=RMS, dtype=BF16, weights=None,
                 layout=BNHD, joint=False, own_pos=False, far=200, freq=None, eps=1e-6, size=1.0, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.args = dict(heads=heads, kv_heads=kv, head_dim=d, axis_dims=dims, theta=theta, inv_freq=freq, norm=norm, eps=eps, dtype=dtype,
                         weight_dtype=weights, layout=layout, pairing=rf2.RF2_ROPE_HALVES if halves else rf2.RF2_ROPE_PAIRS)
        self.plan = rf2.RopePlan(**self.args)
        self.norm, self.eps, self.dtype, self.layout, self.d, self.heads, self.kv = norm, eps, dtype, layout, d, heads, kv
        self.shape = (batch, tokens)
        pos = torch.randint(-far, far + 1, ((batch,) if own_pos else ()) + (tokens, len(dims)), generator=gen, dtype=torch.int64).to(torch.int32)
        self.pos = pos.cuda()
        self.rot = ref.Rotation(pos.numpy() if own_pos else pos.numpy()[None], d, dims, theta, halves, freq)

        def rows(n, parts):
            x = (torch.randn(batch, tokens, n, d, generator=gen) * size * (0.3 + 2 * torch.rand(n, d, generator=gen))).to(dtype).cuda()
            x = x.split(parts, 2)
            return x if layout == BNHD else [y.transpose(1, 2) if joint else y.transpose(1, 2).contiguous() for y in x]

        if joint:
            self.q, self.k, _ = rows(heads + 2 * kv, [heads, kv, kv])
            self.dq_out, self.dk_out, _ = rows(heads + 2 * kv, [heads, kv, kv])
        else:
            (self.q,), (self.k,), (self.dq_out,), (self.dk_out,) = (rows(n, [n]) for n in (heads, kv, heads, kv))
        t = weights or dtype
        self.wq, self.wk = ((1 + 0.3 * torch.randn(d, generator=gen)).to(t).cuda() if norm == RMS else None for _ in range(2))

    def like(self, x):
        return torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda")

    def rows(self, x):
        return f64(x if self.layout == BNHD else x.transpose(1, 2))

    def near(self, got, want, error, what):
        got = self.rows(got)
        off = np.abs(got - want) / ref.rounded(want, error, self.dtype)
        worst, finite = float(off.max()), bool(np.isfinite(got).all())
        assert finite and worst <= 1.0, (what, worst, np.unravel_index(off.argmax(), off.shape))

    def check(self, q_out, k_out):
        for got, x, w, what in ((q_out, self.q, self.wq, "q"), (k_out, self.k, self.wk, "k")):
            if got is not None:
                self.near(got, *ref.forward(self.rot, self.rows(x), None if w is None else f64(w), self.eps), what)

    def forward(self):
        q_out, k_out = self.like(self.q), self.like(self.k)
        self.plan.rf2_rope_apply(self.q, self.k, self.pos, q_out, k_out, self.wq, self.wk)
        self.check(q_out, k_out)
        return q_out, k_out

    def backward(self):
        dq, dk = self.like(self.q), self.like(self.k)
        dw = [torch.full((self.d,), float("nan"), device="cuda") if self.norm == RMS else None for _ in range(2)]
        ws = torch.full((self.plan.info.workspace_bytes,), 255, dtype=torch.uint8, device="cuda") if self.norm == RMS else None
        self.plan.rf2_rope_backward(self.q, self.k, self.pos, self.dq_out, self.dk_out, dq, dk, self.wq, self.wk, *dw, ws)
        for got, got_w, x, dz, w, what in ((dq, dw[0], self.q, self.dq_out, self.wq, "dq"), (dk, dw[1], self.k, self.dk_out, self.wk, "dk")):
            dx, error, want_w, error_w = ref.backward(self.rot, self.rows(x), self.rows(dz), None if w is None else f64(w), self.eps)
            self.near(got, dx, error, what)
            if w is not None:
                off = np.abs(f64(got_w) - want_w) / (error_w + 2.0 ** -24 * np.abs(want_w))
                assert off.max() <= 1.0, (what, "weights", off.max())
        return dq, dk, *dw


CASES = [
    dict(tokens=1), dict(tokens=1, batch=5, own_pos=True), dict(tokens=1, heads=1, kv=1, d=64, dims=(64,)), dict(tokens=2, heads=3, kv=1, d=64, dims=(16, 24, 24)),
    dict(), dict(halves=True), dict(d=64, dims=(16, 24, 24)), dict(d=64, dims=(16, 24, 24), halves=True),
    dict(norm=NONE), dict(norm=NONE, halves=True), dict(norm=NONE, d=64, dims=(64,), halves=True), dict(norm=NONE, d=64, dims=(20, 44)),
    dict(dtype=F16), dict(dtype=F16, halves=True, weights=F32), dict(dtype=F16, norm=NONE), dict(weights=F32), dict(dtype=F16, d=64, dims=(32, 32), halves=True, weights=F32),
    dict(layout=BHND), dict(layout=BHND, halves=True), dict(layout=BHND, d=64, dims=(64,)), dict(layout=BHND, batch=3, own_pos=True, tokens=11),
    dict(joint=True), dict(joint=True, layout=BHND), dict(joint=True, batch=2, tokens=19, d=64, dims=(16, 24, 24)), dict(joint=True, heads=32, kv=8, dims=(128,), halves=True),
    dict(heads=40, kv=40, tokens=130, layout=BHND), dict(heads=40, kv=40, tokens=130), dict(heads=7, kv=7, tokens=65), dict(heads=6, kv=3, d=64, dims=(64,), tokens=513),
    dict(dims=(128,)), dict(dims=(64, 64)), dict(dims=(32, 32, 32, 32)), dict(dims=(0, 2, 0, 40)), dict(dims=(30, 40, 50), halves=True), dict(dims=()), dict(dims=(), d=64, dtype=F16),
    dict(dims=(2,), d=64, halves=True), dict(dims=(126,), halves=True),
    dict(batch=3, tokens=50, own_pos=True), dict(batch=3, tokens=50), dict(batch=2, tokens=333, heads=16, kv=4, d=64, dims=(16, 24, 24), dtype=F16, weights=F32, own_pos=True),
    dict(far=2 ** 31 - 1, tokens=100), dict(far=2 ** 31 - 1, tokens=100, halves=True, norm=NONE, dims=(128,), theta=1e6), dict(far=0),
    dict(theta=100.0), dict(theta=1e-2, dims=(8, 8, 8), far=1000), dict(dims=(6, 4), freq=(1.0, 0.0, -0.3, 65536.0, 1e-9), far=10 ** 6),
    dict(eps=1.0), dict(eps=1e-30), dict(size=1e4), dict(size=1e-3, eps=1e-6), dict(size=1e-3, dtype=F16), dict(size=1000.0, dtype=F16),
    dict(tokens=4099, heads=5, kv=1), dict(tokens=2050, heads=12, kv=12, layout=BHND, dtype=F16), dict(tokens=3001, heads=8, kv=8, d=64, dims=(16, 24, 24), batch=2),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case):
    Case(**case).forward()


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradients(case):
    Case(**case).backward()


@pytest.mark.parametrize("halves", [False, True])
def test_gradients_equal_differences(halves):
    # differences of the loss sum(z dz), taken in 64 bits of the formula: step 1e-4, so they are off by third derivatives of 1e-8 and
    # cancellation of 1e-16 / 1e-4
    c = Case(batch=1, tokens=3, heads=2, kv=1, d=64, dims=(20, 44), halves=halves, dtype=F16, weights=F32, eps=1e-2)
    dq, dk, dwq, dwk = c.backward()
    for x, dz, w, got, got_w in ((c.q, c.dq_out, c.wq, dq, dwq), (c.k, c.dk_out, c.wk, dk, dwk)):
        x, dz, w = c.rows(x), c.rows(dz), f64(w)
        _, error, _, error_w = ref.backward(c.rot, x, dz, w, c.eps)

        def loss(x, w):
            return (ref.forward(c.rot, x, w, c.eps)[0] * dz).sum()

        step = 1e-4
        for i in list(np.ndindex(x.shape))[::5]:
            e = np.zeros_like(x)
            e[i] = step
            want = (loss(x + e, w) - loss(x - e, w)) / (2 * step)
            assert abs(c.rows(got)[i] - want) <= ref.rounded(want, error[i], F16) + 1e-6
        for i in range(64):
            e = np.zeros_like(w)
            e[i] = step
            want = (loss(x, w + e) - loss(x, w - e)) / (2 * step)
            assert abs(f64(got_w)[i] - want) <= error_w[i] + 2.0 ** -24 * abs(want) + 1e-6


@pytest.mark.parametrize("case", [dict(), dict(norm=NONE, layout=BHND), dict(joint=True, tokens=300, heads=16, kv=4), dict(halves=True, d=64, dims=(64,))], ids=str)
def test_outputs_over_inputs(case):
    c = Case(**case)
    want = c.forward()
    q, k = c.q.clone() if not case.get("joint") else c.q, c.k.clone() if not case.get("joint") else c.k
    back = c.backward()
    dq, dk = c.dq_out.clone(), c.dk_out.clone()
    dw = [torch.empty(c.d, device="cuda") if c.norm == RMS else None for _ in range(2)]
    ws = c.plan.alloc_workspace()
    c.plan.rf2_rope_backward(c.q, c.k, c.pos, dq, dk, dq, dk, c.wq, c.wk, *dw, ws)
    for a, b in zip(back, (dq, dk, *dw)):
        assert a is None or torch.equal(a, b)
    c.plan.rf2_rope_apply(q, k, c.pos, q, k, c.wq, c.wk)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("case", [dict(), dict(norm=NONE), dict(tokens=300)], ids=str)
def test_one_side_alone(case):
    c = Case(**case)
    q_out, k_out = c.forward()
    back = c.backward()
    norm = c.norm == RMS
    for side in "qk":
        q, k = (x if side == s else None for s, x in (("q", c.q), ("k", c.k)))
        out = c.like(c.q if side == "q" else c.k)
        c.plan.rf2_rope_apply(q, k, c.pos, out if side == "q" else None, out if side == "k" else None, c.wq if side == "q" else None, c.wk if side == "k" else None)
        assert torch.equal(out, q_out if side == "q" else k_out)
        out, dw = c.like(out), torch.empty(c.d, device="cuda") if norm else None
        pick = lambda s, x: x if side == s else None  # noqa: E731
        c.plan.rf2_rope_backward(q, k, c.pos, pick("q", c.dq_out), pick("k", c.dk_out), pick("q", out), pick("k", out), pick("q", c.wq), pick("k", c.wk),
                                 pick("q", dw), pick("k", dw), c.plan.alloc_workspace() if norm else None)
        assert torch.equal(out, back[0] if side == "q" else back[1])
        assert not norm or torch.equal(dw, back[2] if side == "q" else back[3])


def test_what_lies_between_rows_stays():
    c = Case(tokens=21, heads=3, kv=2, d=64, dims=(64,))
    wide_q, wide_k = (torch.full((1, 21, n + 2, 64 + 16), 7.0, dtype=BF16, device="cuda") for n in (3, 2))
    q_out, k_out = wide_q[:, :, 1:4, 8:72], wide_k[:, :, 1:3, 8:72]
    c.plan.rf2_rope_apply(c.q, c.k, c.pos, q_out, k_out, c.wq, c.wk)
    c.check(q_out, k_out)
    q_out.fill_(7.0), k_out.fill_(7.0)
    assert (wide_q == 7.0).all() and (wide_k == 7.0).all()
    c.plan.rf2_rope_backward(c.q, c.k, c.pos, c.dq_out, c.dk_out, q_out, k_out, c.wq, c.wk, *(torch.empty(64, device="cuda") for _ in range(2)), c.plan.alloc_workspace())
    q_out.fill_(7.0), k_out.fill_(7.0)
    assert (wide_q == 7.0).all() and (wide_k == 7.0).all()


def test_inputs_that_are_broadcast():
    # the gradient of a sum over heads and tokens has strides of 0
    c = Case(tokens=29, heads=5, kv=5)
    one = torch.randn(1, 1, 1, 128, device="cuda").to(BF16)
    c.dq_out = c.dk_out = one.expand(1, 29, 5, 128)
    a = c.backward()
    c.dq_out = c.dk_out = one.expand(1, 29, 5, 128).contiguous()
    assert all(torch.equal(x, y) for x, y in zip(a, c.backward()))
    c.q = c.q[:, :, :1].expand(1, 29, 5, 128)
    c.forward()


def test_nothing_to_do():
    c = Case(tokens=0)
    c.plan.rf2_rope_apply(c.q, c.k, c.pos, c.like(c.q), c.like(c.k), c.wq, c.wk)
    dw = [torch.full((128,), 9.0, device="cuda") for _ in range(2)]
    c.plan.rf2_rope_backward(c.q, c.k, c.pos, c.dq_out, c.dk_out, c.like(c.q), c.like(c.k), c.wq, c.wk, *dw, c.plan.alloc_workspace())
    assert (dw[0] == 0).all() and (dw[1] == 0).all()            # sums over no rows


@pytest.mark.parametrize("batch,tokens", [(0, 5), (2, 0), (0, 0)])
@pytest.mark.parametrize("layout", [BHND, BNHD])
def test_nothing_to_do_with_rows_that_have_an_address(batch, tokens, layout):
    # torch's empty tensors have none; those of other programs may
    plan, at = rf2.RopePlan(heads=4, kv_heads=2, head_dim=128, axis_dims=(128,)), torch.full((4096,), 9.0, dtype=BF16, device="cuda")
    token, head = (128, 128 * 5) if layout == BHND else (128 * 4, 128)
    rows, dw = (at.data_ptr(), 128 * 5 * 4, token, head), [torch.full((128,), 9.0, device="cuda") for _ in range(2)]
    pos, w, workspace = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.ones(128, dtype=BF16, device="cuda"), plan.alloc_workspace()
    stream = torch.cuda.current_stream().cuda_stream
    assert rf2.lib().rf2_rope_apply(plan._h, batch, tokens, rf2.struct.pack("=" + "Qqqq" * 4, *rows * 4), pos.data_ptr(), 0, w.data_ptr(), w.data_ptr(), stream) == 0
    assert rf2.lib().rf2_rope_backward(plan._h, batch, tokens, rf2.struct.pack("=" + "Qqqq" * 6, *rows * 6), pos.data_ptr(), 0, w.data_ptr(), w.data_ptr(),
                                       dw[0].data_ptr(), dw[1].data_ptr(), workspace.data_ptr(), stream) == 0
    assert (at == 9.0).all() and (dw[0] == 0).all() and (dw[1] == 0).all()


def test_rows_of_zeros_and_rows_that_are_not_finite():
    c = Case(tokens=12, heads=2, kv=2)
    c.q[:, 3] = 0
    c.q[:, 5, 0, 17] = float("nan")
    c.q[:, 7, 1, 20] = float("inf")
    c.q[:, 9, 0, 1] = 3e38                                       # squares that 32 bits do not hold
    c.q[:, 10] *= 1e37
    q_out, k_out = c.like(c.q), c.like(c.k)
    c.plan.rf2_rope_apply(c.q, c.k, c.pos, q_out, k_out, c.wq, c.wk)
    assert (q_out[0, 3] == 0).all()
    assert q_out[0, 5, 0].isnan().all()
    row = q_out[0, 7, 1].clone()
    assert row[20:22].isnan().all()
    row[20:22] = 0
    assert (row == 0).all()
    bad = torch.zeros(12, 2, dtype=torch.bool)
    bad[5, 0] = bad[7, 1] = True
    assert q_out[0][~bad.cuda()].isfinite().all() and k_out.isfinite().all()
    c.check(None, k_out)
    c.q[0, bad.cuda()] = 0
    q_out[0, bad.cuda()] = 0
    c.check(q_out, None)
    c.dq_out[:, 9:11] *= 1e30                                    # (the gradients of large rows are small)
    c.backward()


def test_the_same_call_gives_the_same_bits_and_rows_do_not_depend_on_their_batch():
    c = Case(tokens=2000, heads=16, kv=4, d=64, dims=(16, 24, 24))
    a, b = c.backward(), c.backward()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    q_out, k_out = c.forward()
    few = slice(700, 741)
    q_few, k_few = c.like(c.q[:, few]), c.like(c.k[:, few])
    c.plan.rf2_rope_apply(c.q[:, few], c.k[:, few], c.pos[few], q_few, k_few, c.wq, c.wk)
    assert torch.equal(q_few, q_out[:, few]) and torch.equal(k_few, k_out[:, few])


def test_streams_and_graphs():
    c = Case(tokens=777, heads=8, kv=2, joint=True)
    want, back = c.forward(), c.backward()
    q, k, pos = c.q.clone(), c.k.clone(), c.pos.clone()
    out = [c.like(q), c.like(k)]
    grads = [c.like(q), c.like(k), torch.empty(128, device="cuda"), torch.empty(128, device="cuda")]
    dq_out, dk_out, ws = c.dq_out.clone(), c.dk_out.clone(), c.plan.alloc_workspace()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.plan.rf2_rope_apply(q, k, pos, *out, c.wq, c.wk, stream=side)
    side.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])

    def step():
        c.plan.rf2_rope_apply(q, k, pos, *out, c.wq, c.wk)
        c.plan.rf2_rope_backward(q, k, pos, dq_out, dk_out, grads[0], grads[1], c.wq, c.wk, grads[2], grads[3], ws)

    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    with torch.cuda.graph(other):                   # with the same workspace: they run one after the other
        step()
    for rep in range(4):
        for dst, src in ((q, c.q), (k, c.k), (dq_out, c.dq_out)):
            dst.copy_(torch.roll(src, rep, 1))
        pos.copy_(c.pos + rep)
        for t in out + grads:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        (graph, other)[rep % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out + grads]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, out + grads)), rep
        if rep == 0:
            assert all(torch.equal(x, y) for x, y in zip(got, list(want) + list(back)))


def test_two_calls_at_once():
    c, other = Case(tokens=5000, heads=8, kv=8), Case(tokens=5000, heads=8, kv=8, seed=1)
    want = [x.backward() for x in (c, other)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[x.like(x.q), x.like(x.k), torch.empty(128, device="cuda"), torch.empty(128, device="cuda"), x.plan.alloc_workspace()] for x in (c, other)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, s, g in zip((c, other), streams, got):
            x.plan.rf2_rope_backward(x.q, x.k, x.pos, x.dq_out, x.dk_out, g[0], g[1], x.wq, x.wk, g[2], g[3], g[4], stream=s)
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))


def test_offsets_beyond_32_bits():
    # rows of one tensor 6 GB apart; the rows between are never touched
    tokens, heads = 3, 2
    far = 3 * 2 ** 30 // 8 * 8                      # elements
    store = torch.empty(far * (tokens - 1) + 4096, dtype=BF16, device="cuda")
    c = Case(tokens=tokens, heads=heads, kv=1)
    wide = store.as_strided((1, tokens, heads, 128), (0, far, 128, 1))
    wide.copy_(c.q)
    want = c.forward()
    q_out = c.like(c.q)
    c.plan.rf2_rope_apply(wide, c.k, c.pos, q_out, c.like(c.k), c.wq, c.wk)
    assert torch.equal(q_out, want[0])
    c.plan.rf2_rope_apply(wide, c.k, c.pos, wide, c.like(c.k), c.wq, c.wk)
    assert torch.equal(wide, want[0])
    del store, wide


def test_many_rows_of_one_weight():
    # 1.3 million rows: the sums of the weights' gradients
    c = Case(tokens=32760, heads=40, kv=1, seed=3)
    dq, dk, dwq, dwk = (torch.empty_like(c.q), torch.empty_like(c.k), torch.empty(128, device="cuda"), torch.empty(128, device="cuda"))
    c.plan.rf2_rope_backward(c.q, c.k, c.pos, c.dq_out, c.dk_out, dq, dk, c.wq, c.wk, dwq, dwk, c.plan.alloc_workspace())
    cos, sin = (torch.from_numpy(np.ascontiguousarray(x[0])).cuda() for x in (c.rot.cos, c.rot.sin))
    g = torch.empty(32760, 40, 128, dtype=torch.float64, device="cuda")
    dz = c.dq_out[0].double()
    g[..., 0::2] = dz[..., 0::2] * cos[..., 0::2] + dz[..., 1::2] * sin[..., 0::2]
    g[..., 1::2] = dz[..., 1::2] * cos[..., 1::2] - dz[..., 0::2] * sin[..., 1::2]
    x = c.q[0].double()
    n = x / (x.square().mean(-1, keepdim=True) + c.eps).sqrt()
    want, size = (g * n).sum((0, 1)), (g.abs() * n.abs()).sum((0, 1))
    # (terms off by 60 U of their size at most, sums of a token's 40 heads among them, and not all one way: the square root of their number
    # would be 1/1100 of this)
    assert ((dwq.double() - want).abs() <= 60 * ref.U * size + 1e-7 * want.abs()).all()
    assert ((dwq.double() - want).norm() / want.norm()).item() < 1e-5


@pytest.mark.parametrize("tokens, heads, layout", [(1 << 24, 1, BNHD), (1 << 24, 1, BHND), (5, 65535, BNHD), (5, 65535, BHND), (70001, 300, BNHD)], ids=str)
def test_the_largest_sizes(tokens, heads, layout):
    # against calls of a few tokens, bit for bit
    rope = rf2.RopePlan(heads=heads, kv_heads=1, head_dim=64, axis_dims=(40, 20), layout=layout)
    torch.manual_seed(0)
    shape = (tokens, heads, 64) if layout == BNHD else (heads, tokens, 64)
    q = torch.randn(shape, dtype=BF16, device="cuda")
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (tokens, 2), dtype=torch.int32, device="cuda")
    w = torch.randn(64, dtype=BF16, device="cuda")
    out = torch.empty_like(q)
    rope.rf2_rope_apply(q, None, pos, out, None, w)
    few = sorted({0, 1, tokens // 3, tokens // 2 + 1, tokens - 2, tokens - 1})
    for n in few:
        row = q[n:n + 1] if layout == BNHD else q[:, n:n + 1]
        one = torch.empty(row.shape, dtype=BF16, device="cuda")
        rope.rf2_rope_apply(row, None, pos[n:n + 1], one, None, w)
        assert torch.equal(out[n:n + 1] if layout == BNHD else out[:, n:n + 1], one), n
    # gradients: of an output of zeros but for one token, the row's own and nothing else
    dz, dx, dw, dw_one = torch.zeros_like(q), torch.full_like(q, 7.0), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    n = few[-2]
    (dz[n:n + 1] if layout == BNHD else dz[:, n:n + 1]).normal_()
    ws = rope.alloc_workspace()
    rope.rf2_rope_backward(q, None, pos, dz, None, dx, None, w, None, dw, None, ws)
    at = (slice(n, n + 1),) if layout == BNHD else (slice(None), slice(n, n + 1))
    one = torch.empty(dz[at].shape, dtype=BF16, device="cuda")
    rope.rf2_rope_backward(q[at], None, pos[n:n + 1], dz[at], None, one, None, w, None, dw_one, None, ws)
    assert torch.equal(dx[at], one)
    assert int((dx != 0).sum()) == int((one != 0).sum())
    assert torch.allclose(dw, dw_one, rtol=1e-5, atol=1e-5 * dw_one.abs().max().item())          # (sums of up to 65,535 rows in another order)


def test_batches_whose_elements_have_one_token():
    # [batch, 1, heads, d], as a step of single tokens may come, strides of the axis of one of no account
    c = Case(batch=37, tokens=1, heads=8, kv=2, own_pos=True)
    want = c.forward()
    flat = [x.view(37, x.shape[2], 128) for x in (c.q, c.k)]
    out = [torch.empty_like(x) for x in flat]
    c.plan.rf2_rope_apply(flat[0], flat[1], c.pos[:, 0].contiguous(), *out, c.wq, c.wk)
    assert all(torch.equal(a, b[:, 0]) for a, b in zip(out, want))
    odd = c.q.as_strided(c.q.shape, (c.q.stride(0), 3, 128, 1))
    q_out = c.like(c.q)
    c.plan.rf2_rope_apply(odd, None, c.pos, q_out, None, c.wq)
    assert torch.equal(q_out, want[0])
