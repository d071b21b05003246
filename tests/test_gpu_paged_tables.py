"""Pages, slots and rows of a paged cache against loops over the tokens; steps of a program, eager and from a graph."""
import numpy as np
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


class State:
    """A pool with sequences in it, as host lists and on the device."""

    def __init__(self, lens, page, n_pages, row, seed=0, holes=0.0):
        rng = np.random.default_rng(seed)
        order = rng.permutation(n_pages).astype(np.int32)
        self.page, self.n_pages, self.row, self.lens = page, n_pages, row, list(lens)
        self.table = np.full((len(lens), row), -1, dtype=np.int32)
        at = 0
        for s, x in enumerate(lens):
            n = ref.ceil_div(x, page)
            self.table[s, :n] = order[at:at + n]
            at += n
        assert at <= n_pages
        self.free = np.concatenate([order[at:], np.full(at, -7, dtype=np.int32)])
        self.n_free = n_pages - at
        self.table[(rng.random(self.table.shape) < holes) & (self.table >= 0)] = -1

    def plan(self, max_tokens=1, **over):
        args = dict(heads=2, kv_heads=1, head_dim=64, page=self.page, n_pages=self.n_pages, max_seqs=max(1, len(self.lens)),
                    max_pages=self.row, max_tokens=max(1, max_tokens))
        args.update(over)
        return rf2.PagedPlan(**args)

    def append(self, new, n_tokens, in_place=False, n_free=None):
        n_free = self.n_free if n_free is None else n_free
        plan = self.plan(n_tokens)
        want = ref.append(self.lens, new, self.free, n_free, self.table, n_tokens, self.page, self.n_pages)
        table, lens, top = torch.from_numpy(self.table).cuda(), ints(self.lens), ints([n_free])
        lens_out = lens if in_place in (True, "lengths") else ints([-9] * len(self.lens))
        top_out = top if in_place in (True, "count") else ints([-9])
        cu, slots, status = ints([-9] * (len(self.lens) + 1)), ints([-9] * n_tokens), ints([-9])
        free = torch.from_numpy(self.free).cuda()
        plan.rf2_paged_append(lens, ints(new), free, top, table, lens_out, top_out, cu, slots, status)
        got = (table.cpu().numpy(), lens_out.tolist(), top_out.item(), cu.tolist(), slots.tolist(), status.item())
        assert got[5] == want[5], (got[5], want[5])
        assert np.array_equal(got[0], want[0])
        assert got[1:5] == tuple(want[1:5])
        assert np.array_equal(free.cpu().numpy(), self.free)
        return want


@pytest.mark.parametrize("in_place", [False, True, "lengths", "count"])
@pytest.mark.parametrize("page", [32, 64, 256])
@pytest.mark.parametrize("lens, new, pad", [
    ([0], [1], 0), ([31], [1], 0), ([32], [1], 3), ([5, 0, 64, 63], [1, 1, 1, 1], 0), ([0, 0, 0], [0, 0, 0], 4), ([], [], 5),
    ([100, 0, 7], [0, 300, 65], 1), ([10, 500], [700, 4000], 100), ([3], [9000], 0),
], ids=str)
def test_append(lens, new, pad, page, in_place):
    row = max([ref.ceil_div(x + n, page) for x, n in zip(lens, new)] + [1])
    need = sum(ref.ceil_div(x + n, page) for x, n in zip(lens, new))
    State(lens, page, need + 2, row, seed=page).append(new, sum(new) + pad, in_place)
    State(lens, page, max(1, need), row + 3, seed=page + 1).append(new, sum(new) + pad, in_place)


@pytest.mark.parametrize("n_seqs, most", [(1000, 3), (1025, 30), (4096, 2), (130, 200)])
def test_append_many_sequences(n_seqs, most):
    rng = np.random.default_rng(n_seqs)
    lens, new = rng.integers(0, 100, n_seqs).tolist(), rng.integers(0, most, n_seqs).tolist()
    for in_place in (False, True):
        State(lens, 32, 12000, 12, seed=1).append(new, sum(new) + 11, in_place)


@pytest.mark.parametrize("n_tokens_less, n_free, lens, new, row", [
    (1, None, [5, 6], [1, 1], 2), (0, 0, [32, 6], [1, 1], 2), (0, 1, [32, 32], [1, 1], 2), (0, None, [5, 6], [1, -1], 2),
    (0, None, [63, 6], [2, 1], 2), (0, -1, [5, 6], [1, 1], 2), (0, 10 ** 6, [5, 6], [1, 1], 2), (0, 0, [32, 6], [5000, 1], 200),
    (3, 0, [63, 6], [2, -4], 2), (0, None, [5, 6], [2 ** 31 - 1, 2 ** 31 - 1], 2),
], ids=str)
def test_append_refuses_as_a_whole(n_tokens_less, n_free, lens, new, row):
    tokens = min(max(0, sum(new)) - n_tokens_less, 6000)
    want = State(lens, 32, 300, row, seed=4).append(new, tokens, n_free=n_free)
    assert want[5] != 0
    State(lens, 32, 300, row, seed=4).append(new, tokens, in_place=True, n_free=n_free)


def test_append_behind_a_hole_gives_no_slots_there():
    st = State([40, 40], 32, 10, 4, seed=2)
    st.table[0, 1] = -1
    want = st.append([30, 2], 32)
    assert want[4][:24] == [-1] * 24 and min(want[4][24:]) >= 0


@pytest.mark.parametrize("holes", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("n_seqs, longest, share", [(1, 40, 1.0), (7, 2000, 0.5), (300, 900, 0.4), (3, 400000, 1.0), (64, 300, 0.0), (4096, 40, 0.7)])
def test_release(n_seqs, longest, share, holes):
    rng = np.random.default_rng(n_seqs)
    lens = rng.integers(0, longest, n_seqs).tolist()
    page = 32
    held = sum(ref.ceil_div(x, page) for x in lens)
    for in_place in (False, True):
        st = State(lens, page, held + 5, ref.ceil_div(longest, page) + 1, seed=5, holes=holes)
        done = (rng.random(n_seqs) < share).tolist()
        want = ref.release(done, st.lens, st.table, st.free, st.n_free, page, st.n_pages)
        table, free, top, lens_d, status = torch.from_numpy(st.table).cuda(), torch.from_numpy(st.free).cuda(), ints([st.n_free]), ints(lens), ints([-9])
        lens_out, top_out = (lens_d, top) if in_place else (ints([-9] * n_seqs), ints([-9]))
        st.plan().rf2_paged_release(torch.tensor(done, device="cuda"), lens_d, table, free, top, lens_out, top_out, status)
        assert status.item() == want[3] == 0
        assert np.array_equal(free.cpu().numpy(), np.array(want[0]))
        assert lens_out.tolist() == want[1] and top_out.item() == want[2]
        assert np.array_equal(table.cpu().numpy(), st.table)


@pytest.mark.parametrize("lens, n_free, code", [([40, 40], 18, ref.POOL_FULL), ([-1, 40], 2, ref.BAD_LENGTH), ([40, 97], 2, ref.BAD_LENGTH),
                                                ([40, 40], -1, ref.BAD_LENGTH), ([40, 40], 21, ref.BAD_LENGTH)], ids=str)
def test_release_refuses_as_a_whole(lens, n_free, code):
    st = State([40, 40], 32, 20, 3, seed=5)
    table, free, status = torch.from_numpy(st.table).cuda(), torch.from_numpy(st.free).cuda(), ints([-9])
    lens_out, top_out = ints([-9] * 2), ints([-9])
    st.plan().rf2_paged_release(torch.tensor([1, 1], dtype=torch.uint8, device="cuda"), ints(lens), table, free, ints([n_free]), lens_out, top_out, status)
    assert status.item() == code and lens_out.tolist() == lens and top_out.item() == n_free
    assert np.array_equal(free.cpu().numpy(), st.free)


def test_release_counts_holes_where_every_entry_would_be_too_many():
    """20 pages, 18 said to be free, 4 entries given back: too many, unless two of them are holes."""
    st = State([40, 40], 32, 20, 3, seed=5)
    st.table[0, 0] = st.table[1, 1] = -1
    want = ref.release([True, True], st.lens, st.table, st.free, 18, 32, 20)
    free, lens_out, top_out, status = torch.from_numpy(st.free).cuda(), ints([0, 0]), ints([0]), ints([-9])
    st.plan().rf2_paged_release(torch.tensor([True, True], device="cuda"), ints(st.lens), torch.from_numpy(st.table).cuda(), free, ints([18]), lens_out, top_out, status)
    assert want[3] == status.item() == 0 and top_out.item() == 20 and np.array_equal(free.cpu().numpy(), np.array(want[0]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("kv, d, page", [(1, 64, 32), (8, 128, 64), (3, 128, 256), (5, 64, 128)])
@pytest.mark.parametrize("kind", ["run", "offset", "reversed", "scattered", "one", "skipped"])
def test_store(kind, kv, d, page, dtype):
    gen = torch.Generator().manual_seed(kv + d)
    n_pages = 11
    size = n_pages * page
    slots = {"run": list(range(page, page + 97)), "offset": list(range(13, 13 + 130)), "reversed": list(range(200, 100, -1)),
             "scattered": torch.randperm(size, generator=gen)[:75].tolist(), "one": [size - 1],
             "skipped": [-1, 5, 6, 7, size, 8, 9, -2 ** 31, 2 ** 31 - 1, 10, 11, 4] + list(range(32, 60)) + [-1]}[kind]
    n = len(slots)
    plan = rf2.PagedPlan(heads=kv, kv_heads=kv, head_dim=d, page=page, n_pages=n_pages, max_seqs=1, max_pages=1, max_tokens=200, dtype=dtype)
    buf = plan.alloc()
    buf["k_cache"].fill_(3.0)
    buf["v_cache"].fill_(4.0)
    k_want, v_want = buf["k_cache"].cpu(), buf["v_cache"].cpu()
    joint = torch.randn(n, 3 * kv, d, generator=gen).to(dtype)
    _, k, v = joint.cuda().split(kv, 1)
    if kind in ("offset", "one"):
        k, v = k.contiguous(), v.contiguous()
    plan.rf2_paged_store(k, v, ints(slots), buf["k_cache"], buf["v_cache"])
    ref.put(k_want, v_want, [s if 0 <= s < size else -1 for s in slots], k.cpu(), v.cpu(), page)
    assert torch.equal(buf["k_cache"].cpu().view(torch.int16), k_want.view(torch.int16))
    assert torch.equal(buf["v_cache"].cpu().view(torch.int16), v_want.view(torch.int16))


@pytest.mark.parametrize("seed", range(6))
def test_store_of_many_sequences(seed):
    """Runs of neighbouring slots as appends leave them, of random lengths from random places of pages in random order; some are -1."""
    rng = np.random.default_rng(seed)
    page, kv, d, n_pages = int(rng.choice([32, 64, 128, 256])), int(rng.choice([1, 3, 8])), int(rng.choice([64, 128])), 40
    order, slots = rng.permutation(n_pages), []
    for p in order[:25]:
        first, n = int(rng.integers(0, page)), int(rng.choice([1, 2, 7, 31, 32, 33, 300]))
        slots += [int(p) * page + r for r in range(first, min(page, first + n))]
        slots += [-1] * int(rng.choice([0, 0, 0, 1, 40]))
    plan = rf2.PagedPlan(heads=kv, kv_heads=kv, head_dim=d, page=page, n_pages=n_pages, max_seqs=1, max_pages=1, max_tokens=len(slots))
    buf = plan.alloc()
    buf["k_cache"].fill_(3.0)
    buf["v_cache"].fill_(4.0)
    k_want, v_want = buf["k_cache"].cpu(), buf["v_cache"].cpu()
    k, v = torch.randn(len(slots), 2 * kv, d, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda().split(kv, 1)
    plan.rf2_paged_store(k, v, ints(slots), buf["k_cache"], buf["v_cache"])
    ref.put(k_want, v_want, slots, k.cpu(), v.cpu(), page)
    assert torch.equal(buf["k_cache"].cpu().view(torch.int16), k_want.view(torch.int16))
    assert torch.equal(buf["v_cache"].cpu().view(torch.int16), v_want.view(torch.int16))


def test_store_of_the_same_slot_twice_leaves_one_of_the_two():
    plan = rf2.PagedPlan(heads=1, kv_heads=1, head_dim=64, page=32, n_pages=2, max_seqs=1, max_pages=1, max_tokens=64)
    buf = plan.alloc()
    k = torch.randn(10, 1, 64, device="cuda").to(torch.bfloat16)
    slots = [0, 1, 2, 3, 2, 40, 41, 42, 43, 41]
    plan.rf2_paged_store(k, k, ints(slots), buf["k_cache"], buf["v_cache"])
    for slot, at in ((2, (2, 4)), (41, (6, 9))):
        P, r = slot // 32, slot % 32
        got = (buf["k_cache"][P, 0, 0, :, r].reshape(64), buf["v_cache"][P, 0, 0, r // 16 * 2 + r % 8 // 4, :, r % 16 // 8 * 4 + r % 4])
        for x in got:
            assert ((x == k[at[0], 0]) | (x == k[at[1], 0])).all()


def test_store_past_32_bits():
    n_pages = 9000
    plan = rf2.PagedPlan(heads=8, kv_heads=8, head_dim=128, page=256, n_pages=n_pages, max_seqs=1, max_pages=1, max_tokens=64)
    buf = plan.alloc()
    last = n_pages * 256 - 40
    k, v = (torch.randn(40, 8, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    plan.rf2_paged_store(k, v, ints(range(last, last + 40)), buf["k_cache"], buf["v_cache"])
    want_k, want_v = buf["k_cache"][-1:].clone().zero_(), buf["v_cache"][-1:].clone().zero_()
    ref.put_many(want_k, want_v, torch.arange(216, 256, device="cuda"), k, v, 256)
    there = want_k != 0
    assert torch.equal(buf["k_cache"][-1:][there], want_k[there])
    there = want_v != 0
    assert torch.equal(buf["v_cache"][-1:][there], want_v[there])


# ---- steps of a program ---------------------------------------------------------------------------------------------

class Server:
    """A small model's worth of state: two layers' caches over one set of tables, and every row ever stored on the host."""

    def __init__(self, max_seqs=6, causal=True, dtype=torch.bfloat16, seed=0):
        self.page, self.kv, self.heads, self.d, self.seqs, self.dtype = 32, 2, 4, 64, max_seqs, dtype
        self.plan = rf2.PagedPlan(heads=4, kv_heads=2, head_dim=64, page=32, n_pages=64, max_seqs=max_seqs, max_pages=16, max_tokens=256,
                                  dtype=dtype, causal=causal)
        self.buf = self.plan.alloc()
        self.caches = [(self.buf["k_cache"].fill_(float("nan")), self.buf["v_cache"].fill_(float("nan"))),
                       (self.buf["k_cache"].clone(), self.buf["v_cache"].clone())]
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rows = [[(torch.empty(0, 2, 64, device="cuda", dtype=dtype),) * 2 for _ in range(max_seqs)] for _ in self.caches]
        self.causal = causal

    def inputs(self, n):
        return [[torch.randn(n, h, 64, generator=self.gen, device="cuda").to(self.dtype) for h in (4, 2, 2)] for _ in self.caches]

    def launch(self, new, step, qkv, outs):
        b, p = self.buf, self.plan
        p.rf2_paged_append(b["seq_len"], new, b["free_pages"], b["n_free"], b["block_table"], b["seq_len"], b["n_free"], step["cu_new"],
                           step["slots"], b["status"])
        for (k_cache, v_cache), (q, k, v), o in zip(self.caches, qkv, outs):
            p.rf2_paged_store(k, v, step["slots"], k_cache, v_cache)
            p.rf2_paged_attn(q, k_cache, v_cache, b["block_table"], b["seq_len"], step["cu_new"], b["workspace"], o)

    def release(self, done):
        b = self.buf
        self.plan.rf2_paged_release(torch.tensor(done, device="cuda"), b["seq_len"], b["block_table"], b["free_pages"], b["n_free"],
                                    b["seq_len"], b["n_free"], b["status"])
        assert b["status"].item() == 0
        for rows in self.rows:
            for s, d in enumerate(done):
                if d:
                    rows[s] = (rows[s][0][:0], rows[s][1][:0])

    def check(self, new, qkv, outs, pad):
        assert self.buf["status"].item() == 0
        half = torch.finfo(self.dtype).eps / 2
        for layer, ((q, k, v), o) in enumerate(zip(qkv, outs)):
            at = 0
            for s, n in enumerate(new):
                old = self.rows[layer][s]
                ks, vs = torch.cat([old[0], k[at:at + n]]), torch.cat([old[1], v[at:at + n]])
                self.rows[layer][s] = (ks, vs)
                want, _, tol, _ = ref.attention(q[at:at + n], ks, vs, torch.ones(len(ks), dtype=torch.bool, device="cuda"), n, self.causal, 0.125, half)
                assert ((o[at:at + n].double() - want).abs() <= tol).all(), (layer, s)
                at += n
            assert (o[at:] == 7.0).all() and len(o) == at + pad
        assert self.buf["seq_len"].tolist() == [len(r[0]) for r in self.rows[0]]


STEPS = [([40, 0, 33, 5, 0, 0], 2), ([1, 64, 1, 1, 0, 1], 0), ([1, 1, 1, 1, 0, 1], 3), "release", ([1, 1, 30, 1, 90, 1], 1), ([1, 1, 1, 1, 1, 1], 0),
         "release", ([100, 1, 1, 60, 1, 1], 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_steps_of_a_program(causal, dtype):
    srv = Server(causal=causal, dtype=dtype)
    done = iter([[False, False, True, False, False, True], [True, False, False, True, False, False]])
    for step in STEPS:
        if step == "release":
            srv.release(next(done))
            continue
        new, pad = step
        n = sum(new) + pad
        qkv = srv.inputs(n)
        bufs = srv.plan.alloc_step(srv.seqs, n)
        outs = [torch.full_like(bufs["o"], 7.0) for _ in qkv]
        srv.launch(ints(new), bufs, qkv, outs)
        srv.check(new, qkv, outs, pad)
    held = sum(ref.ceil_div(x, 32) for x in srv.buf["seq_len"].tolist())
    assert srv.buf["n_free"].item() == 64 - held
    pages = srv.buf["free_pages"][:64 - held].tolist()
    for s, x in enumerate(srv.buf["seq_len"].tolist()):
        pages += srv.buf["block_table"][s, :ref.ceil_div(x, 32)].tolist()
    assert sorted(pages) == list(range(64))


def test_a_step_replays_from_a_graph_with_other_lengths():
    srv = Server(seed=3)
    n = 40
    new, qkv, step = ints([0] * 6), srv.inputs(n), srv.plan.alloc_step(6, n)
    outs = [torch.full_like(step["o"], 7.0) for _ in qkv]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        srv.launch(new, step, qkv, outs)               # (no new tokens: nothing changes)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        srv.launch(new, step, qkv, outs)
    for lens in ([30, 4, 0, 1, 0, 5], [1, 1, 1, 1, 1, 1], [0, 0, 40, 0, 0, 0], [1, 1, 1, 1, 1, 0], [2, 9, 3, 0, 20, 6]):
        new.copy_(ints(lens))
        for layer, fresh in zip(qkv, srv.inputs(n)):
            for dst, src in zip(layer, fresh):
                dst.copy_(src)
        for o in outs:
            o.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        srv.check(lens, qkv, outs, n - sum(lens))


def test_a_step_that_does_not_fit_does_nothing():
    srv = Server(seed=4)
    first = srv.inputs(200)
    step = srv.plan.alloc_step(6, 200)
    outs = [torch.full_like(step["o"], 7.0) for _ in first]
    srv.launch(ints([200, 0, 0, 0, 0, 0]), step, first, outs)
    srv.check([200, 0, 0, 0, 0, 0], first, outs, 0)
    before = [x.clone() for pair in srv.caches for x in pair] + [srv.buf[k].clone() for k in ("block_table", "seq_len", "free_pages", "n_free")]
    for o in outs:
        o.fill_(7.0)
    srv.launch(ints([150, 0, 0, 30, 0, 21]), step, srv.inputs(200), outs)         # 201 tokens for 200 rows
    assert srv.buf["status"].item() == rf2.RF2_PAGED_TOKENS_FULL
    srv.launch(ints([1, -1, 0, 0, 0, 0]), step, srv.inputs(200), outs)
    assert srv.buf["status"].item() == rf2.RF2_PAGED_BAD_LENGTH
    after = [x for pair in srv.caches for x in pair] + [srv.buf[k] for k in ("block_table", "seq_len", "free_pages", "n_free")]
    for x, y in zip(before, after):
        assert torch.equal(x.view(torch.int16) if x.is_floating_point() else x, y.view(torch.int16) if y.is_floating_point() else y)
    assert all((o == 7.0).all() for o in outs)


def test_a_call_can_be_taken_back():
    """Outputs apart from the inputs: the same step again gives the same pages."""
    st = State([10, 70], 32, 12, 6, seed=9)
    first = st.append([40, 5], 45)
    again = st.append([40, 5], 45)
    assert np.array_equal(first[0], again[0]) and first[1:] == again[1:]
