"""The layer's permutation with Q and K normalised and rotated on the way: against the two calls one after the other (bit for bit), block means
against the formulas in 64 bits, the whole layer."""
import numpy as np
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests import rope_ref as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
BHND, BNHD = rf2.RF2_LAYOUT_BHND, rf2.RF2_LAYOUT_BNHD


class Case:
    def __init__(self, *, batch=1, heads=5, d=128, T=5, H=10, W=13, block=128, block_k=0, sink=1, text=0, layout=BHND, dims=(44, 42, 42), halves=False,
                 norm=rf2.RF2_NORM_RMS, weights=None, own_pos=False, text_weights=True, cdf=None, sparsity=0.5, seed=0, sink_at_end=1):
        gen = torch.Generator().manual_seed(seed)
        self.plan = rf2.Plan(batch=batch, heads=heads, head_dim=d, T=T, H=H, W=W, block=block, block_k=block_k, sparsity=sparsity, sink_frames=sink,
                             text_tokens=text, qkv_layout=layout, cdf_threshold=cdf, sink_at_end=sink_at_end)
        self.rope = rf2.RopePlan(heads=heads, kv_heads=heads, head_dim=d, axis_dims=dims, norm=norm, weight_dtype=weights, layout=layout,
                                 pairing=rf2.RF2_ROPE_HALVES if halves else rf2.RF2_ROPE_PAIRS)
        self.layout, self.halves, self.dims, self.norm, self.d = layout, halves, dims, norm == rf2.RF2_NORM_RMS, d
        n = self.n = T * H * W + text
        self.video = T * H * W
        shape = (batch, heads, n, d) if layout == BHND else (batch, n, heads, d)

        def rows():
            return (torch.randn(shape, generator=gen) * (0.3 + 2 * torch.rand(d, generator=gen))).to(BF16).cuda()

        self.q, self.k, self.v = rows(), rows(), rows()
        grid = torch.stack(torch.meshgrid(*(torch.arange(x) for x in (T, H, W)), indexing="ij"), -1).view(-1, 3)
        pos = torch.cat([grid, T + torch.arange(text)[:, None].expand(-1, 3)])[:, 3 - len(dims):] if len(dims) <= 3 else torch.cat([grid, grid[:, :1]], 1)
        self.pos = (torch.stack([pos + 5 * b for b in range(batch)]) if own_pos else pos).int().contiguous().cuda()
        t = weights or BF16
        weight = lambda: (1 + 0.3 * torch.randn(d, generator=gen)).to(t).cuda()  # noqa: E731
        self.w = [weight(), weight()] if self.norm else [None, None]
        self.w_text = [weight(), weight()] if self.norm and text and text_weights else [None, None]

    def tokens(self, x, begin, end):
        return x[:, :, begin:end] if self.layout == BHND else x[:, begin:end]

    def prepared(self):
        """q and k after rf2_rope_apply: the grid's tokens and the text with weights of their own."""
        q, k = torch.empty_like(self.q), torch.empty_like(self.k)
        cut = self.video if self.w_text[0] is not None else self.n
        for begin, end, w in ((0, cut, self.w), (cut, self.n, self.w_text)):
            if end > begin:
                self.rope.rf2_rope_apply(self.tokens(self.q, begin, end), self.tokens(self.k, begin, end), self.pos[..., begin:end, :].contiguous(),
                                         self.tokens(q, begin, end), self.tokens(k, begin, end), *w)
        return q, k

    def permute(self, buf, q=None, k=None, v=None, **over):
        self.plan.rf2_permute_rope(self.rope, self.q if q is None else q, self.k if k is None else k, self.v if v is None else v, self.pos,
                                   buf["qp"], buf["kp"], buf["vp"], buf["qbar"], buf["kbar"], *self.w, *self.w_text, **over)

    def means(self, x, w, w_text, b, tb, perm):
        """Block means in 64 bits and how far 32 bits may be: an error of each row, and sums of up to b numbers."""
        x = (x if self.layout == BNHD else x.transpose(1, 2)).cpu().double().numpy()
        pos = self.pos.cpu().numpy()
        rot = ref.Rotation(pos if pos.ndim == 3 else pos[None], self.d, self.dims, halves=self.halves)
        if w is not None:
            w = np.tile(w.cpu().double().numpy(), (self.n, 1, 1))
            if w_text is not None:
                w[self.video:] = w_text.cpu().double().numpy()
        z, error = ref.forward(rot, x, w)
        out = []
        for y in (z[:, perm], error[:, perm], np.abs(z[:, perm])):
            y = np.concatenate([y, np.zeros((y.shape[0], tb * b - self.n) + y.shape[2:])], 1)
            y = y.reshape(y.shape[0], tb, b, *y.shape[2:]).sum(2).transpose(0, 2, 1, 3)
            count = np.full(tb, b)
            count[-1] = self.n - (tb - 1) * b
            out.append(y / count[:, None])
        return out[0], out[1] + (b // 32 + 8) * ref.U * out[2]


def filled(plan):
    buf = plan.alloc("cuda")
    for t in buf.values():
        t.fill_(-77)
    return buf


CASES = [
    dict(), dict(halves=True), dict(norm=rf2.RF2_NORM_NONE), dict(norm=rf2.RF2_NORM_NONE, halves=True, d=64, dims=(64,), layout=BNHD),
    dict(layout=BNHD), dict(layout=BNHD, halves=True, weights=F32), dict(d=64, dims=(16, 24, 24)), dict(d=64, dims=(16, 24, 24), halves=True, layout=BNHD),
    dict(block=64), dict(block=64, block_k=128), dict(block=128, block_k=64, layout=BNHD), dict(block=256, block_k=128), dict(block=256, block_k=64, d=64, dims=(64,)),
    dict(text=17), dict(text=17, text_weights=False), dict(text=200, layout=BNHD, halves=True), dict(text=130, sink=0, d=64, dims=(64,), weights=F32), dict(text=1, norm=rf2.RF2_NORM_NONE),
    dict(batch=2, heads=3), dict(batch=3, heads=4, own_pos=True, layout=BNHD), dict(heads=1), dict(heads=8, T=1, H=16, W=16, sink=0, dims=(64, 64)), dict(heads=2, T=1, H=1, W=1, sink=0),
    dict(T=1, H=3, W=5, sink=0, d=64, dims=(30, 34)), dict(T=2, H=7, W=9, sink=1, sink_at_end=0), dict(dims=(126,), halves=True), dict(dims=()), dict(dims=(8, 16, 32, 64)),
    dict(T=9, H=20, W=26, heads=12, layout=BNHD), dict(T=9, H=20, W=26, heads=12),                                  # 45 MB and more
    dict(T=13, H=30, W=26, heads=14), dict(T=13, H=30, W=26, heads=24, d=64, dims=(16, 24, 24), layout=BNHD), dict(T=21, H=30, W=26, heads=13, text=33),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_equals_the_two_calls_and_its_means_the_formulas(case):
    c = Case(**case)
    buf, want = filled(c.plan), filled(c.plan)
    c.permute(buf)
    c.plan.rf2_permute(*c.prepared(), c.v, want["qp"], want["kp"], want["vp"], want["qbar"], want["kbar"])
    for name in ("qp", "kp", "vp"):
        assert torch.equal(buf[name].view(torch.int16), want[name].view(torch.int16)), name
    perm, _ = c.plan.rf2_plan_perm()
    i = c.plan.info
    for name, x, w, w_text, b, tb in (("qbar", c.q, c.w[0], c.w_text[0], c.plan.cfg.block, i.n_blocks), ("kbar", c.k, c.w[1], c.w_text[1], i.block_k, i.n_blocks_k)):
        mean, error = c.means(x, w, w_text, b, tb, perm)
        off = np.abs(buf[name].cpu().double().numpy() - mean) / (error + 2.0 ** -140)
        worst = float(off.max())
        assert worst <= 1.0, (name, worst)
    c.plan.rf2_permute_rope(c.rope, c.q, c.k, c.v, c.pos, want["qp"].zero_(), want["kp"].zero_(), want["vp"].zero_(), None, None, *c.w, *c.w_text)
    for name in ("qp", "kp", "vp"):                                # without means
        assert torch.equal(buf[name].view(torch.int16), want[name].view(torch.int16)), name


@pytest.mark.parametrize("halves", [False, True])
def test_rows_behind_the_last_are_zeros_whatever_the_weights_are(halves):
    # 850 tokens of which the last 200 are text: the last block has 82 rows of text and 46 behind them
    c = Case(text=200, halves=halves)
    want, buf = filled(c.plan), filled(c.plan)
    c.permute(want)
    c.w = [torch.full_like(w, float("inf")) for w in c.w]
    c.permute(buf)
    for name in ("qbar", "kbar"):
        got, last = buf[name].view(5, -1, 128), want[name].view(5, -1, 128)[:, -1]
        assert torch.equal(got[:, -1], last) and not got[:, 0].isfinite().any(), name
    assert torch.equal(buf["qp"].view(5, -1, 128, 128)[:, -1], want["qp"].view(5, -1, 128, 128)[:, -1])
    assert torch.equal(buf["kp"].view(5, -1, 128, 128)[:, -1], want["kp"].view(5, -1, 128, 128)[:, -1])


@pytest.mark.parametrize("layout", [BHND, BNHD])
def test_outputs_over_inputs(layout):
    # kp over q, vp over k, as for a caller short of memory: three launches, the same values (16 blocks, none partly filled)
    c = Case(T=4, H=16, W=32, heads=6, layout=layout, sink=0)
    want, buf = filled(c.plan), filled(c.plan)
    c.permute(want)
    q, k = c.q.clone(), c.k.clone()
    buf["kp"], buf["vp"] = q.view(-1)[:buf["kp"].numel()].view(buf["kp"].shape), k.view(-1)[:buf["vp"].numel()].view(buf["vp"].shape)
    c.permute(buf, q=q, k=k)
    for name in ("qp", "kp", "vp", "qbar", "kbar"):
        assert torch.equal(buf[name], want[name]), name


@pytest.mark.parametrize("case", [dict(T=6, H=16, W=16), dict(T=6, H=16, W=16, text=40, layout=BNHD, halves=True), dict(T=6, H=16, W=16, cdf=0.8)], ids=str)
def test_the_layer_on_raw_projections(case):
    c = Case(**case)
    buf = c.plan.alloc("cuda", scores=True)
    o = c.plan.layer_fused(c.q, c.k, c.v, buf, rope=c.rope, pos=c.pos, weights=(*c.w, *(w for w in c.w_text if w is not None))).clone()
    # the attention of the lists it made, on rows of the two calls
    q, k = c.prepared()
    other = c.plan.alloc("cuda", scores=True)
    c.plan.rf2_permute(q, k, c.v, other["qp"], other["kp"], other["vp"], other["qbar"], other["kbar"])
    c.plan.rf2_block_sparse_attn_unpermuted(other["qp"], other["kp"], other["vp"], buf["blk_idx"], buf["blk_cnt"], other["o"])
    assert torch.equal(o, other["o"])
    # and its scores are theirs but for the rounding of rows to bf16: means of 128 of them, half a step each, with random signs; a dot product of d
    c.plan.rf2_predict_mask(other["qbar"], other["kbar"], other["blk_idx"], other["blk_cnt"], None, other["scores"])
    a, b = buf["scores"].double(), other["scores"].double()
    assert (a - b).abs().max() <= 0.02 * b.abs().max()
    # everything kept: the same layer bit for bit
    dense = Case(**dict(case, cdf=None, sparsity=0.0))
    buf = dense.plan.alloc("cuda")
    o = dense.plan.layer_fused(c.q, c.k, c.v, buf, rope=c.rope, pos=c.pos, weights=(*c.w, *(w for w in c.w_text if w is not None))).clone()
    assert torch.equal(o, dense.plan.layer_fused(q, k, c.v, buf))


def test_graph():
    c = Case(text=17, heads=6, layout=BNHD)
    buf, eager = c.plan.alloc("cuda"), c.plan.alloc("cuda")
    weights = (*c.w, *c.w_text)
    base, pos = [x.clone() for x in (c.q, c.k, c.v)], c.pos.clone()
    c.plan.layer_fused(c.q, c.k, c.v, buf, rope=c.rope, pos=c.pos, weights=weights)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.plan.layer_fused(c.q, c.k, c.v, buf, rope=c.rope, pos=c.pos, weights=weights)
    for rep in range(4):
        for dst, src in zip((c.q, c.k, c.v), base):
            dst.copy_(torch.roll(src, rep, 2))
        c.pos.copy_(pos + 7 * rep)
        buf["o"].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.plan.layer_fused(c.q, c.k, c.v, eager, rope=c.rope, pos=c.pos, weights=weights)
        torch.cuda.synchronize()
        assert torch.equal(buf["o"], eager["o"]) and torch.equal(buf["blk_idx"], eager["blk_idx"]) and torch.equal(buf["qbar"], eager["qbar"]), rep


def test_offsets_beyond_32_bits():
    # 4.6 GB and 2.3e9 elements a tensor, token-major: rows of late tokens and heads lie behind both limits
    heads, T, H, W = 150, 33, 45, 80
    plan = rf2.Plan(batch=1, heads=heads, head_dim=128, T=T, H=H, W=W, block=128, sparsity=0.8, sink_frames=1, qkv_layout=BNHD)
    rope = rf2.RopePlan(heads=heads, kv_heads=heads, head_dim=128, axis_dims=(44, 42, 42))
    n = T * H * W
    torch.manual_seed(0)
    q, k, v = (torch.randn(1, n, heads, 128, dtype=BF16, device="cuda") for _ in range(3))
    pos = torch.randint(0, 100, (n, 3), dtype=torch.int32, device="cuda")
    w = [torch.randn(128, dtype=BF16, device="cuda") for _ in range(2)]
    got, want = plan.alloc("cuda"), plan.alloc("cuda")
    plan.rf2_permute_rope(rope, q, k, v, pos, got["qp"], got["kp"], got["vp"], got["qbar"], got["kbar"], *w)
    rope.rf2_rope_apply(q, k, pos, q, k, *w)
    plan.rf2_permute(q, k, v, want["qp"], want["kp"], want["vp"], want["qbar"], want["kbar"])
    for name in ("qp", "kp", "vp"):
        assert torch.equal(got[name], want[name]), name
    for name in ("qbar", "kbar"):                              # rows before and behind their rounding: half a step of up to 8, averaged
        assert (got[name] - want[name]).abs().max() < 2.0 ** -6, name
    perm, _ = plan.rf2_plan_perm()
    last = torch.from_numpy(perm[-300:].astype(np.int64)).cuda()
    assert torch.equal(got["qp"][0, -1, n - 300:n], q[0, last, -1])
