"""New tokens of a paged cache normalised, rotated and stored in one call: against the two calls one after the other, bit for bit, and a program's
steps."""
import pytest
import torch

from paper_2512_24086_amd import rf2

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


class Case:
    def __init__(self, *, tokens=37, heads=8, kv=2, d=128, page=64, dims=(44, 42, 42), halves=False, norm=rf2.RF2_NORM_RMS, dtype=BF16, weights=None, joint=False,
                 start=5, n_pages=None, seed=0):
        gen = torch.Generator().manual_seed(seed)
        n_pages = n_pages or (tokens + start) // page + 5
        self.plan = rf2.PagedPlan(heads=heads, kv_heads=kv, head_dim=d, page=page, n_pages=n_pages, max_seqs=4, max_pages=n_pages, max_tokens=max(1, tokens), dtype=dtype)
        self.rope = rf2.RopePlan(heads=heads, kv_heads=kv, head_dim=d, axis_dims=dims, norm=norm, dtype=dtype, weight_dtype=weights,
                                 pairing=rf2.RF2_ROPE_HALVES if halves else rf2.RF2_ROPE_PAIRS)
        self.tokens, self.heads, self.kv, self.d, self.dtype = tokens, heads, kv, d, dtype
        parts = [heads, kv, kv]
        x = (torch.randn(tokens, sum(parts), d, generator=gen) * (0.3 + 2 * torch.rand(d, generator=gen))).to(dtype).cuda()
        self.q, self.k, self.v = x.split(parts, 1) if joint else (y.contiguous() for y in x.split(parts, 1))
        self.pos = torch.randint(0, 100000, (tokens, len(dims)), generator=gen).int().cuda()
        t = weights or dtype
        self.w = [(1 + 0.3 * torch.randn(d, generator=gen)).to(t).cuda() if norm == rf2.RF2_NORM_RMS else None for _ in range(2)]
        # slots: a run from `start` on through pages in any order
        order = torch.randperm(n_pages, generator=gen)
        at = torch.arange(tokens) + start
        self.slots = (order[at // page] * page + at % page).int().cuda()

    def cache(self):
        shape = (self.plan.cfg.n_pages, self.kv, self.plan.cfg.page // 32)
        return (torch.full((*shape, self.d // 8, 32, 8), 3.0, dtype=self.dtype, device="cuda"), torch.full((*shape, 4, self.d, 8), 5.0, dtype=self.dtype, device="cuda"))

    def both(self, cu_new=None, live=None, slots=None):
        slots = self.slots if slots is None else slots
        live = self.tokens if live is None else live
        q_out, caches = torch.full((self.tokens, self.heads, self.d), 7.0, dtype=self.dtype, device="cuda"), self.cache()
        self.plan.rf2_paged_store_rope(self.rope, self.q, self.k, self.v, self.pos, slots, *caches, q_out, *self.w, cu_new=cu_new)
        q_want, k_want, cache_want = torch.full_like(q_out, 7.0), torch.empty(self.tokens, self.kv, self.d, dtype=self.dtype, device="cuda"), self.cache()
        self.rope.rf2_rope_apply(self.q[:live], None, self.pos[:live], q_want[:live], None, self.w[0])
        self.rope.rf2_rope_apply(None, self.k, self.pos, None, k_want, None, self.w[1])
        self.plan.rf2_paged_store(k_want, self.v, slots, *cache_want)
        assert torch.equal(q_out, q_want)
        assert torch.equal(caches[0], cache_want[0]) and torch.equal(caches[1], cache_want[1])
        return q_out, caches


@pytest.mark.parametrize("case", [
    dict(), dict(tokens=1), dict(tokens=2, heads=1, kv=1, d=64, dims=(64,)), dict(halves=True), dict(norm=rf2.RF2_NORM_NONE), dict(norm=rf2.RF2_NORM_NONE, halves=True, d=64, dims=(64,)),
    dict(d=64, dims=(16, 24, 24)), dict(dtype=F16), dict(dtype=F16, halves=True, weights=F32, dims=(128,)), dict(dtype=F16, d=64, dims=(32, 32)), dict(weights=F32),
    dict(joint=True), dict(joint=True, heads=32, kv=8, tokens=100, dims=(128,), halves=True), dict(page=32, tokens=131), dict(page=256, tokens=300, start=250), dict(heads=40, kv=40, tokens=97),
    dict(tokens=1000, heads=12, kv=4, d=64, dims=(16, 24, 24), joint=True), dict(tokens=64, dims=()), dict(tokens=4680, heads=10, kv=10, joint=True, start=1), dict(tokens=33, kv=8, heads=8, start=31),
], ids=str)
def test_equals_the_two_calls(case):
    Case(**case).both()


@pytest.mark.parametrize("slots", ["run", "single", "threes", "backwards", "mixed"])
@pytest.mark.parametrize("tokens,kv,d", [(8, 8, 128), (9, 8, 128), (48, 8, 128), (256, 8, 128), (257, 8, 128), (48, 40, 128), (49, 40, 128), (256, 8, 64), (264, 8, 64), (2048, 1, 128),
                                         (2049, 1, 64)])
def test_workgroups_of_few_and_of_many_tokens(tokens, kv, d, slots):
    # V is stored eight tokens to a workgroup up to 256 workgroups: both sides, with keys of V that go out whole and one by one
    c = Case(tokens=tokens, heads=kv, kv=kv, d=d, dims=(d,), n_pages=tokens // 4 + 6)
    i = torch.arange(tokens)
    order = torch.randperm(c.plan.cfg.n_pages, generator=torch.Generator().manual_seed(1))
    if slots == "single":                                     # sixteen keys apart
        at = i * 16 + 5
    elif slots == "threes":
        at = i // 3 * 32 + i % 3 + 7
    elif slots == "backwards":
        at = tokens + 20 - i
    else:
        at = i + 5
    at = order[at // 64] * 64 + at % 64
    if slots == "mixed":                                      # a third of a run is padding
        at = torch.where(torch.rand(tokens, generator=torch.Generator().manual_seed(2)) < 0.3, -1, at)
    c.both(slots=at.int().cuda())


@pytest.mark.parametrize("slots", ["run", "runs", "single", "backwards", "padding", "anything"])
@pytest.mark.parametrize("tokens,kv,d,halves", [(700, 48, 128, False), (1025, 33, 128, True), (999, 40, 64, False), (4099, 8, 64, True)])
def test_wavefronts_that_begin_where_lines_do(tokens, kv, d, halves, slots):
    # K in large calls, whose wavefronts take 1 to 15 tokens: each of them once, wherever runs begin and end
    c = Case(tokens=tokens, heads=kv, kv=kv, d=d, dims=(d,), halves=halves, page=32, n_pages=tokens // 4 + 8)
    gen = torch.Generator().manual_seed(tokens)
    i, order = torch.arange(tokens), torch.randperm(c.plan.cfg.n_pages, generator=gen)
    if slots == "runs":                                       # of 1 to 40 tokens, up to 16 slots apart
        step = torch.ones(tokens, dtype=torch.long)
        at = 0
        while (at := at + int(torch.randint(1, 41, (), generator=gen))) < tokens:
            step[at] = int(torch.randint(1, 17, (), generator=gen))
        at = step.cumsum(0) + 2
    else:
        at = {"run": i + 13, "single": i * 8 + i % 8, "backwards": tokens + 9 - i, "padding": i + 3, "anything": torch.randperm(4 * tokens, generator=gen)[:tokens]}[slots]
    at = order[at // 32] * 32 + at % 32
    if slots == "padding":                                    # and slots that the cache does not have
        bad = torch.tensor([-1, -8, c.plan.cfg.n_pages * 32, 2 ** 31 - 1, -2 ** 31])
        at = torch.where(torch.rand(tokens, generator=gen) < 0.2, bad[torch.randint(0, 5, (tokens,), generator=gen)], at)
    c.both(slots=at.int().cuda())


@pytest.mark.parametrize("live", [0, 1, 30, 50])
def test_padding_stays(live):
    c = Case(tokens=50)
    cu_new = torch.tensor([0, live // 2, live], dtype=torch.int32, device="cuda")
    slots = c.slots.clone()
    slots[live:] = -1
    q_out, _ = c.both(cu_new, live, slots)
    assert (q_out[live:] == 7.0).all()


@pytest.mark.parametrize("count", [-5, 51, 2 ** 31 - 1, -2 ** 31])
def test_counts_out_of_range_are_clamped(count):
    c = Case(tokens=50)
    c.both(torch.tensor([count], dtype=torch.int32, device="cuda"), 0 if count < 0 else 50)


def test_slots_out_of_range_are_left_out_of_the_cache_alone():
    c = Case(tokens=50)
    slots = c.slots.clone()
    slots[3], slots[17], slots[49] = -1, c.plan.cfg.n_pages * 64, 2 ** 31 - 1
    c.both(slots=slots)                                       # Q of these tokens is rotated all the same


def test_q_over_itself_and_slices_of_a_wider_tensor():
    c = Case(tokens=45, joint=True)
    q_want, caches_want = c.both()
    wide = torch.full((45, 8 * 128 + 64), 9.0, dtype=BF16, device="cuda")
    out = wide[:, 32:32 + 1024].view(45, 8, 128)
    c.plan.rf2_paged_store_rope(c.rope, c.q, c.k, c.v, c.pos, c.slots, *c.cache(), out, *c.w)
    assert torch.equal(out, q_want) and (wide[:, :32] == 9.0).all() and (wide[:, -32:] == 9.0).all()
    caches = c.cache()
    c.plan.rf2_paged_store_rope(c.rope, c.q, c.k, c.v, c.pos, c.slots, *caches, c.q, *c.w)
    assert torch.equal(c.q, q_want) and all(torch.equal(a, b) for a, b in zip(caches, caches_want))


def test_no_tokens():
    c = Case(tokens=0)
    caches = c.cache()
    c.plan.rf2_paged_store_rope(c.rope, c.q, c.k, c.v, c.pos, c.slots, *caches, c.q, *c.w)
    assert (caches[0] == 3.0).all() and (caches[1] == 5.0).all()


def test_steps_of_a_program_eager_and_from_a_graph():
    # prompts, then single tokens: tables, then Q, K and V of two layers, then attention; against a program that rotates by itself
    heads, kv, d, page, room = 8, 2, 64, 32, 300
    plan = rf2.PagedPlan(heads=heads, kv_heads=kv, head_dim=d, page=page, n_pages=64, max_seqs=3, max_pages=40, max_tokens=room)
    rope = rf2.RopePlan(heads=heads, kv_heads=kv, head_dim=d, axis_dims=(d,), pairing=rf2.RF2_ROPE_HALVES, theta=1e6)
    torch.manual_seed(5)
    w = [(1 + 0.3 * torch.randn(d)).to(BF16).cuda() for _ in range(2)]

    class Program:
        def __init__(self, fused):
            self.fused, self.s = fused, plan.alloc()
            self.layers = [(self.s["k_cache"].zero_(), self.s["v_cache"].zero_()), (torch.zeros_like(self.s["k_cache"]), torch.zeros_like(self.s["v_cache"]))]
            self.new_len, self.step = torch.zeros(3, dtype=torch.int32, device="cuda"), plan.alloc_step(3, room)
            self.x, self.pos = torch.zeros(room, heads + 2 * kv, d, dtype=BF16, device="cuda"), torch.zeros(room, 1, dtype=torch.int32, device="cuda")
            self.o = [torch.zeros(room, heads, d, dtype=BF16, device="cuda") for _ in range(2)]

        def run(self):
            s, t = self.s, self.step
            plan.rf2_paged_append(s["seq_len"], self.new_len, s["free_pages"], s["n_free"], s["block_table"], s["seq_len"], s["n_free"], t["cu_new"], t["slots"], s["status"])
            for (kc, vc), o in zip(self.layers, self.o):
                q, k, v = self.x.split([heads, kv, kv], 1)
                q_out = torch.zeros(room, heads, d, dtype=BF16, device="cuda")
                if self.fused:
                    plan.rf2_paged_store_rope(rope, q, k, v, self.pos, t["slots"], kc, vc, q_out, *w, cu_new=t["cu_new"])
                else:
                    k_out = torch.empty(room, kv, d, dtype=BF16, device="cuda")
                    rope.rf2_rope_apply(q, k, self.pos, q_out, k_out, *w)
                    plan.rf2_paged_store(k_out, v, t["slots"], kc, vc)
                plan.rf2_paged_attn(q_out, kc, vc, s["block_table"], s["seq_len"], t["cu_new"], s["workspace"], o)

    fused, plain, graphed = Program(True), Program(False), Program(True)
    graph = None
    lens = [0, 0, 0]
    for i, new in enumerate([(100, 31, 64), (1, 1, 1), (1, 1, 1), (33, 1, 0), (1, 1, 1)]):
        x = torch.randn(room, heads + 2 * kv, d).to(BF16).cuda()
        pos = torch.zeros(room, 1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(new):
            pos[at:at + n, 0] = torch.arange(lens[s], lens[s] + n)
            at += n
            lens[s] += n
        for p in (fused, plain, graphed):
            p.x.copy_(x), p.pos.copy_(pos), p.new_len.copy_(torch.tensor(new))
            for o in p.o:
                o.fill_(7.0)
        torch.cuda.synchronize()
        fused.run(), plain.run()
        if i == 0:
            graphed.run()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            saved = {n: t.clone() for n, t in graphed.s.items() if n not in ("k_cache", "v_cache")}
            with torch.cuda.graph(graph):
                graphed.run()
            for n, t in saved.items():
                graphed.s[n].copy_(t)
        else:
            graph.replay()
        torch.cuda.synchronize()
        for p in (plain, graphed):
            for a, b in zip(fused.o + [t for pair in fused.layers for t in pair], p.o + [t for pair in p.layers for t in pair]):
                assert torch.equal(a, b), (i, "plain" if p is plain else "graph")
        for o in fused.o:
            assert (o[at:] == 7.0).all() and o[:at].isfinite().all()


def test_offsets_beyond_32_bits():
    # a cache of 5.2e9 elements, tokens in its last pages
    c = Case(tokens=40, heads=8, kv=8, page=256, n_pages=20000)
    size = c.plan.info.cache_elements
    assert size > 2 ** 32
    k_cache, v_cache = torch.zeros(size, dtype=BF16, device="cuda"), torch.zeros(size, dtype=BF16, device="cuda")
    slots = (c.plan.cfg.n_pages * 256 - 1 - 3 * torch.arange(40)).int().cuda()
    q_out, k_want = torch.empty_like(c.q), torch.empty_like(c.k)
    c.plan.rf2_paged_store_rope(c.rope, c.q, c.k, c.v, c.pos, slots, k_cache, v_cache, q_out, *c.w)
    c.rope.rf2_rope_apply(None, c.k, c.pos, None, k_want, None, c.w[1])
    r = slots.long() % 256
    page = slots.long() // 256
    k = k_cache.view(-1, 8, 8, 16, 32, 8)[page, :, r // 32, :, r % 32]
    v = v_cache.view(-1, 8, 8, 4, 128, 8)[page, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4]
    assert torch.equal(k.reshape(40, 8, 128), k_want) and torch.equal(v, c.v)
    assert int((k_cache != 0).sum()) <= 40 * 8 * 128 and int((v_cache != 0).sum()) <= 40 * 8 * 128
