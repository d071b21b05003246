"""Attention of new tokens over a paged cache against its definition in 64 bits, through the C ABI.

The cache is filled with NaN where no token lies, so every test checks too that nothing of it reaches a result."""
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16

CASES = {
    # one token: the shortest caches, odd lengths, ends inside a tile and on its borders
    "one_key": dict(new=[1], ctx=[0], heads=1, kv=1, d=64, page=32),
    "one_d128": dict(new=[1], ctx=[200], heads=8, kv=8, d=128, page=32),
    "borders": dict(new=[1] * 8, ctx=[30, 31, 32, 62, 63, 64, 95, 127], heads=4, kv=2, d=64, page=64),
    "borders_128": dict(new=[1] * 8, ctx=[30, 31, 32, 62, 63, 64, 95, 127], heads=4, kv=2, d=128, page=128, dtype=FP),
    # heads: shared by odd numbers, by more than a tile of rows, none shared
    "group_3": dict(new=[1, 1, 1], ctx=[700, 5, 1300], heads=9, kv=3, d=128, page=64),
    "group_7": dict(new=[1, 2], ctx=[450, 81], heads=7, kv=1, d=64, page=64, dtype=FP),
    "group_40": dict(new=[1, 3], ctx=[600, 10], heads=40, kv=1, d=128, page=32),
    "group_512": dict(new=[1, 2, 0, 1], ctx=[900, 33, 5, 0], heads=512, kv=1, d=64, page=32),
    "mha_512": dict(new=[1, 3], ctx=[1500, 31], heads=512, kv=512, d=64, page=64, dtype=FP),
    "mha_24": dict(new=[1, 1], ctx=[99, 1001], heads=24, kv=24, d=64, page=256),
    # long caches: cut into parts, whole ones beside them
    "long": dict(new=[1], ctx=[20011], heads=8, kv=2, d=128, page=64),
    "long_fp16": dict(new=[1, 1, 1], ctx=[9000, 17, 3333], heads=16, kv=8, d=128, page=128, dtype=FP),
    "million": dict(new=[1], ctx=[1000000], heads=2, kv=1, d=64, page=256),
    "long_d64": dict(new=[1, 1], ctx=[12345, 600], heads=4, kv=4, d=64, page=32),
    # chunks
    "chunk_small": dict(new=[5], ctx=[0], heads=2, kv=1, d=64, page=32),
    "chunk": dict(new=[300], ctx=[77], heads=4, kv=2, d=128, page=64),
    "chunk_fp16": dict(new=[513], ctx=[1000], heads=8, kv=8, d=128, page=128, dtype=FP),
    "chunk_d64": dict(new=[257], ctx=[64], heads=12, kv=4, d=64, page=32),
    "chunk_group_11": dict(new=[2900], ctx=[100], heads=11, kv=1, d=64, page=64),
    "chunk_long": dict(new=[130], ctx=[6000], heads=8, kv=8, d=128, page=64),
    "prompts": dict(new=[200, 1, 77, 640, 33], ctx=[0, 500, 31, 129, 2000], heads=8, kv=2, d=128, page=32),
    "prompts_d64": dict(new=[200, 1, 77, 640, 33], ctx=[0, 500, 31, 129, 2000], heads=16, kv=8, d=64, page=256, dtype=FP),
    # sequences without new tokens, without keys; padding; parts of a joint projection
    "empty_seqs": dict(new=[0, 3, 0, 1, 0], ctx=[50, 0, 0, 640, 7], heads=4, kv=4, d=64, page=32),
    "padded": dict(new=[1, 40, 2], ctx=[100, 20, 3], heads=6, kv=2, d=128, page=64, pad=17),
    "joint": dict(new=[33, 1], ctx=[100, 20], heads=6, kv=2, d=64, page=64, pad=1, fused=True),
    # more sequences than a wavefront has lanes
    "many_seqs": dict(new=[1] * 150, ctx=[(37 * i) % 301 for i in range(150)], heads=4, kv=2, d=64, page=32),
    "many_mixed": dict(new=[(i % 7 == 3) * 40 + i % 3 for i in range(100)], ctx=[(91 * i) % 500 for i in range(100)], heads=4, kv=1, d=128, page=64),
    "more_seqs": dict(new=[i % 3 for i in range(700)], ctx=[(91 * i) % 700 for i in range(700)], heads=4, kv=2, d=64, page=32),
    "more_seqs_long": dict(new=[1] * 300, ctx=[(977 * i) % 60 + 9000 * (i % 150 == 7) for i in range(300)], heads=8, kv=8, d=128, page=64, dtype=FP),
    "more_mixed": dict(new=[(i % 7 == 3) * 140 + i % 3 for i in range(300)], ctx=[(91 * i) % 900 for i in range(300)], heads=8, kv=2, d=128, page=64, pad=5),
    "more_chunks": dict(new=[20 + i % 9 for i in range(270)], ctx=[(i * 131) % 300 for i in range(270)], heads=3, kv=3, d=64, page=64),
    # single tokens of long sequences beside chunks
    "mixed": dict(new=[1, 300, 1, 1, 2, 90, 1, 0, 1, 5, 1, 1], ctx=[3000, 700, 20, 9000, 5, 0, 1, 60, 4100, 333, 2500, 31], heads=8, kv=2, d=128, page=64, pad=3),
    "mixed_d64": dict(new=[1, 1, 260, 1, 1, 1, 130, 1, 1], ctx=[5000, 2100, 900, 64, 63, 0, 2000, 3000, 1500], heads=4, kv=4, d=64, page=32, dtype=FP),
    "mixed_group_20": dict(new=[1, 1, 60, 1, 1, 1, 30, 1, 1], ctx=[5000, 2100, 900, 64, 63, 0, 2000, 3000, 1500], heads=20, kv=1, d=128, page=128),
    "chunks_alone": dict(new=[64, 40, 90, 33, 70, 50, 41, 65, 77], ctx=[600, 0, 900, 64, 63, 10, 2000, 30, 1500], heads=4, kv=4, d=64, page=64),
}


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("name", list(CASES))
def test_attention_matches_the_definition(name, causal):
    b = Batch(seed=len(name), **CASES[name])
    plan = b.plan(causal)
    o, lse = b.run(plan)
    share = b.check(o, lse, causal)
    print(f"{name} causal={causal}: {share:.3f} of the tolerance")
    o2, _ = b.run(plan, with_lse=False)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)), "the same call, the same bits"


@pytest.mark.parametrize("scale", [0.01, 0.5, 3.0])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_scales(dtype, scale):
    """Logits from flat to far apart (with 3.0 the largest decides alone, and references move at most units)."""
    b = Batch(seed=3, new=[1, 50], ctx=[900, 300], heads=4, kv=2, d=64, page=32, dtype=dtype)
    o, lse = b.run(b.plan(scale=scale))
    assert torch.isfinite(o[:b.total].float()).all()
    if scale < 3.0:
        b.check(o, lse, scale=scale)
    else:
        # logits of up to 100: what a logit is off in fp32 goes into the tolerance the same way, apart from the constant for logits below 8
        half = torch.finfo(dtype).eps / 2
        at = 0
        for s, n in enumerate(b.new):
            from tests.paged_ref import attention
            want, want_lse, tol, _ = attention(b.q[at:at + n], b.k[s].cuda(), b.v[s].cuda(), b.kept[s].cuda(), n, True, scale, half)
            assert ((o[at:at + n].double() - want).abs() <= tol + 2.0 ** -15 * b.v[s].abs().max().item()).all()
            at += n


def test_growing_logits_move_the_reference():
    """Keys whose logits grow by a few octaves a unit, over more octaves than either type carries."""
    for dtype in (BF, FP):
        b = Batch(seed=5, new=[1, 20], ctx=[640, 640], heads=2, kv=1, d=64, page=32, dtype=dtype)
        for s in (0, 1):
            grow = torch.linspace(0, 1, b.len[s])[:, None, None]
            b.k[s] = (b.k[s].float() * 0.05 + grow * 30).to(dtype)
            pos = torch.arange(b.len[s])
            slots = b.table[s].cpu()[pos // 32].long() * 32 + pos % 32
            from tests.paged_ref import put_many
            k_cache, v_cache = b.k_cache.cpu(), b.v_cache.cpu()
            put_many(k_cache, v_cache, slots, b.k[s], b.v[s], 32)
            b.k_cache.copy_(k_cache)
        b.q.copy_(b.q.abs() * 0.5)
        o, lse = b.run(b.plan())
        half = torch.finfo(dtype).eps / 2
        at = 0
        for s, n in enumerate(b.new):
            from tests.paged_ref import attention
            want, want_lse, tol, lse_tol = attention(b.q[at:at + n], b.k[s].cuda(), b.v[s].cuda(), b.kept[s].cuda(), n, True, 0.125, half)
            # (logits up to 100 in place of 8: 2^-16 of a probability more)
            assert ((o[at:at + n].double() - want).abs() <= tol + 2.0 ** -15 * b.v[s].abs().max().item()).all()
            assert ((lse[at:at + n].double() - want_lse).abs() <= lse_tol + 2.0 ** -15).all()
            at += n


def test_small_probabilities_count_in_fp16():
    """One key a thousand times as likely as each of 20,000 others: the others' 95 % are not lost to the type."""
    b = Batch(seed=6, new=[1], ctx=[20000], heads=1, kv=1, d=64, page=64, dtype=FP)
    b.q.zero_()
    b.q[:, :, 0] = 1.0
    k = torch.zeros(b.len[0], 1, 64)
    k[0, 0, 0] = 8 * 6.9
    b.k[0] = k.to(FP)
    pos = torch.arange(b.len[0])
    slots = b.table[0].cpu()[pos // 64].long() * 64 + pos % 64
    from tests.paged_ref import put_many
    k_cache, v_cache = b.k_cache.cpu(), b.v_cache.cpu()
    put_many(k_cache, v_cache, slots, b.k[0], b.v[0], 64)
    b.k_cache.copy_(k_cache)
    o, lse = b.run(b.plan())
    b.check(o, lse)


def test_holes_in_the_table_are_left_out():
    marks = [-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1]
    holes = [(0, 0, -1), (0, 3, marks[1]), (1, 1, marks[2])] + [(2, p, marks[p % 4]) for p in range(12)] + [(3, p, -1) for p in range(1, 180)]
    for causal in (True, False):
        for d, dtype in ((64, BF), (128, FP)):
            b = Batch(seed=7, new=[1, 70, 2, 40], ctx=[400, 130, 379, 5800], heads=4, kv=2, d=d, page=32, dtype=dtype, holes=holes)
            o, lse = b.run(b.plan(causal))
            b.check(o, lse, causal)


def test_holes_beside_chunks_and_single_tokens():
    holes = [(s, p, -1) for s in range(9) for p in range(1, 1 + 3 * s)] + [(1, 0, 10 ** 6)]
    for d, dtype, page in ((64, FP, 128), (128, BF, 32)):
        b = Batch(seed=17, new=[1, 1, 200, 1, 1, 1, 150, 1, 1], ctx=[30 * page] * 9, heads=8, kv=4, d=d, page=page, dtype=dtype, holes=holes)
        o, lse = b.run(b.plan())
        b.check(o, lse)
        b = Batch(seed=18, new=[1] * 9, ctx=[30 * page + 5] * 9, heads=8, kv=4, d=d, page=page, dtype=dtype, holes=holes)
        o, lse = b.run(b.plan())
        b.check(o, lse)


def test_a_sequence_of_holes_alone_yields_zeros():
    b = Batch(seed=8, new=[1, 1], ctx=[99, 300], heads=4, kv=2, d=64, page=32, holes=[(0, p, -1) for p in range(4)])
    o, lse = b.run(b.plan())
    assert (o[0] == 0).all() and torch.isinf(lse[0]).all() and (lse[0] < 0).all()
    b.check(o, lse)


def test_lengths_shorter_than_the_chunk_leave_rows_without_keys():
    """seq_len counts fewer tokens than are new: the first tokens stand before the first key."""
    b = Batch(seed=9, new=[10], ctx=[0], heads=2, kv=2, d=64, page=32)
    b.seq_len.fill_(4)
    o, lse = b.run(b.plan())
    assert (o[:6] == 0).all() and torch.isinf(lse[:6]).all()
    b.k[0], b.v[0], b.kept[0] = b.k[0][:4], b.v[0][:4], b.kept[0][:4]
    from tests.paged_ref import attention
    want, want_lse, tol, _ = attention(b.q, b.k[0].cuda(), b.v[0].cuda(), b.kept[0].cuda(), 10, True, 0.125, 2.0 ** -8)
    assert ((o.double() - want).abs() <= tol).all()


def test_lengths_out_of_range_are_clamped():
    b = Batch(seed=10, new=[2, 2], ctx=[60, 62], heads=2, kv=1, d=64, page=32, extra_row=0, fill=0.5)
    plan = b.plan()
    good, _ = b.run(plan)
    b.seq_len[1] = 2 ** 31 - 1               # taken as the row's 64 tokens
    o, _ = b.run(plan)
    assert torch.equal(o, good)
    b.seq_len[1] = -5                        # no keys
    o, lse = b.run(plan)
    assert (o[2:] == 0).all() and torch.isinf(lse[2:]).all() and torch.equal(o[:2], good[:2])
    b.cu.copy_(torch.tensor([-3, 2, 10 ** 9]))
    b.seq_len.fill_(64)
    b.run(plan)
    torch.cuda.synchronize()


@pytest.mark.parametrize("n", [3, 70, 300])
def test_rows_that_overlap_are_refused_by_the_kernel(n):
    """cu_new goes up and down, so that the sequences' rows are together more than there are."""
    b = Batch(seed=16, new=[30] + [0] * n, ctx=[2000] + [1000] * n, heads=8, kv=4, d=64, page=32)
    plan = b.plan()
    b.cu.copy_(torch.tensor([0, 30] * ((n + 2) // 2) + [0] * (n % 2)))
    o, lse = b.run(plan)
    torch.cuda.synchronize()
    assert (o == 7.0).all() and (lse == 7.0).all()


def test_values_that_are_not_finite_stay_with_their_rows():
    """NaN in a row of q; an infinite value of V, which every row that sees it gets."""
    b = Batch(seed=11, new=[3, 1], ctx=[64, 500], heads=4, kv=2, d=64, page=32)
    b.q[1, 2] = float("nan")
    o, _ = b.run(b.plan())
    assert torch.isnan(o[1, 2].float()).all()
    keep = torch.ones(4, 4, dtype=torch.bool)
    keep[1, 2] = False
    assert torch.isfinite(o.float()).all(2)[keep].all()


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", [dict(new=[6, 3], ctx=[40, 61], heads=4, kv=2, d=64), dict(new=[6, 3], ctx=[40, 61], heads=4, kv=2, d=128),
                                   dict(new=[20, 9], ctx=[700, 13], heads=2, kv=2, d=128), dict(new=[150, 70], ctx=[0, 90], heads=4, kv=2, d=64),
                                   dict(new=[150, 70], ctx=[333, 0], heads=4, kv=2, d=128), dict(new=[300], ctx=[2000], heads=1, kv=1, d=128),
                                   dict(new=[300], ctx=[2000], heads=1, kv=1, d=64)], ids=str)
def test_tokens_behind_that_are_not_finite_stay_unseen(shape, dtype):
    """K and V of some new tokens hold infinities and NaN: tokens before them get the bits that they get with zeros there, and from
    them on V's go through as the sum has them (a channel with both infinities, or with a NaN, is not a number)."""
    b = Batch(seed=20, page=64, dtype=dtype, **shape)
    plan = b.plan()
    places = {0: (3, 5), 1: (1, 2)}                       # sequence -> tokens of its chunk
    inf, nan = float("inf"), float("nan")
    values = [(0, inf), (1, -inf), (2, nan), (3, inf)]

    def write(s, pos, ch, v=None, k=None):
        page, r = int(b.table[s, pos // 64]), pos % 64
        if v is not None:
            b.v_cache[page, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, ch, r % 16 // 8 * 4 + r % 4] = v
        if k is not None:
            b.k_cache[page, :, r // 32, ch // 8, r % 32, ch % 8] = k

    for s, (first, second) in list(places.items())[:len(b.new)]:
        for ch, _ in values:
            for t in (first, second):
                write(s, b.ctx[s] + t, ch, v=0.0)
    clean, _ = b.run(plan)
    for s, (first, second) in list(places.items())[:len(b.new)]:
        for ch, x in values:
            write(s, b.ctx[s] + first, ch, v=x)
        write(s, b.ctx[s] + second, 3, v=-inf)             # channel 3: both
    o, _ = b.run(plan)
    at = 0
    for s, n in enumerate(b.new):
        first, second = places[s]
        got, want = o[at:at + n], clean[at:at + n]
        assert torch.equal(got[:first].view(torch.int16), want[:first].view(torch.int16)), s
        assert torch.equal(got[:, :, 4:].contiguous().view(torch.int16), want[:, :, 4:].contiguous().view(torch.int16)), s
        seen = got[first:].float()
        assert (seen[:, :, 0] == inf).all() and (seen[:, :, 1] == -inf).all() and torch.isnan(seen[:, :, 2]).all(), s
        assert (got[first:second, :, 3].float() == inf).all() and torch.isnan(got[second:, :, 3].float()).all(), s
        at += n
    # K of one token: all channels of the tokens from it on.  A row that is out of range makes the rows of its wavefront move their
    # references, so those before it may be rounded otherwise: they are held to the definition, like every result.
    from tests.paged_ref import attention
    for s, (first, second) in list(places.items())[:len(b.new)]:
        for ch, _ in values:
            for t in (first, second):
                write(s, b.ctx[s] + t, ch, v=0.0)
                b.v[s][b.ctx[s] + t, :, ch] = 0.0
    for x in (nan, inf):
        for s in range(len(b.new)):
            write(s, b.ctx[s] + places[s][0], 7, k=x)
        o, _ = b.run(plan)
        at = 0
        for s, n in enumerate(b.new):
            first = places[s][0]
            want, _, tol, _ = attention(b.q[at:at + n], b.k[s].cuda(), b.v[s].cuda(), b.kept[s].cuda(), n, True, 1 / b.d ** 0.5, torch.finfo(dtype).eps / 2)
            assert ((o[at:at + first].double() - want[:first]).abs() <= tol[:first]).all(), s
            if x != inf:
                assert torch.isnan(o[at + first:at + n].float()).all(), s
            at += n


@pytest.mark.parametrize("n", [1, 63, 64, 65, 200, 256, 257, 1024, 1025, 4096])
def test_numbers_of_sequences(n):
    b = Batch(seed=12, new=[1] * n, ctx=[(i * 53) % 90 for i in range(n)], heads=2, kv=1, d=64, page=32)
    o, lse = b.run(b.plan())
    b.check(o, lse)


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB a cache: pages at its end."""
    page, kv, d = 256, 8, 128
    n_pages = 9000                            # 8 GiB less a little each for K and V: 256 * 8 * 128 * 2 bytes a page
    assert n_pages * page * kv * d * 2 > 1 << 32
    b = Batch(seed=13, new=[1, 40], ctx=[1500, 300], heads=16, kv=kv, d=d, page=page)
    k_cache = torch.empty(n_pages, *b.k_cache.shape[1:], dtype=BF, device="cuda")
    v_cache = torch.empty(n_pages, *b.v_cache.shape[1:], dtype=BF, device="cuda")
    shift = n_pages - b.n_pages
    k_cache[shift:], v_cache[shift:] = b.k_cache, b.v_cache
    b.k_cache, b.v_cache = k_cache, v_cache
    b.table = torch.where(b.table >= 0, b.table + shift, b.table)
    o, lse = b.run(b.plan(n_pages=n_pages))
    b.check(o, lse)


def test_more_columns_than_a_wavefront_lists_at_a_time():
    """Parts of more than 512 pages (many rows) and of more than 256 to a wavefront (few), with holes near where a list ends."""
    holes = [(0, p, -1) for p in (0, 255, 256, 511, 512, 513, 560)]
    b = Batch(seed=19, new=[1024], ctx=[17000], heads=128, kv=1, d=64, page=32, holes=holes)
    o, lse = b.run(b.plan(False))
    b.check(o, lse, False)

    n = 128
    b = Batch(seed=20, new=[1], ctx=[35199], heads=8, kv=8, d=64, page=32, holes=[(0, p, -1) for p in (1, 255, 256, 274, 275, 276, 530, 531, 1099)])
    b.new, b.len, b.rows = [1] * n, b.len * n, n
    b.k, b.v, b.kept = b.k * n, b.v * n, b.kept * n                    # all sequences read the same pages
    b.table, b.seq_len = b.table.repeat(n, 1).contiguous(), b.seq_len.repeat(n)
    b.cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    b.q = torch.randn(n, 8, 64, generator=torch.Generator().manual_seed(20)).to(BF).cuda()
    o, lse = b.run(b.plan())
    b.check(o, lse)


def test_streams_and_workspaces():
    """Calls of two streams at a time, a workspace each; a call on a stream that is not the current one."""
    b = Batch(seed=14, new=[1, 1], ctx=[9000, 4000], heads=8, kv=2, d=128, page=64)
    plan = b.plan()
    want, _ = b.run(plan)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [plan.alloc_workspace() for _ in streams]
    outs = [torch.zeros_like(want) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, ws, o in zip(streams, spaces, outs):
            plan.rf2_paged_attn(b.q, b.k_cache, b.v_cache, b.table, b.seq_len, b.cu, ws, o, None, st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_two_graphs_share_a_workspace():
    """Captured calls of different batches, the same workspace, replayed in turn beside eager calls: none keeps anything in it."""
    batches = [Batch(seed=16, new=[1, 1, 1], ctx=[9000, 4000, 10], heads=8, kv=2, d=128, page=64),
               Batch(seed=17, new=[300, 2], ctx=[2000, 700], heads=8, kv=2, d=128, page=64)]
    plans = [b.plan() for b in batches]
    wants = [b.run(p)[0] for b, p in zip(batches, plans)]
    space = plans[0].alloc_workspace()
    outs = [torch.zeros_like(w) for w in wants]

    def call(i):
        b = batches[i]
        plans[i].rf2_paged_attn(b.q, b.k_cache, b.v_cache, b.table, b.seq_len, b.cu, space, outs[i])

    graphs = []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            call(i)
        graphs.append(graph)
    for turn in (0, 1, 1, 0, "eager", 1, 0):
        for o in outs:
            o.zero_()
        for i in ((0, 1) if turn == "eager" else (turn,)):
            call(i) if turn == "eager" else graphs[i].replay()
            assert torch.equal(outs[i], wants[i])


def test_sequences_that_share_pages():
    """A prompt's pages in the rows of several sequences: each reads them as its own."""
    b = Batch(seed=18, new=[1, 1, 3, 1], ctx=[1000, 1040, 1100, 7], heads=8, kv=2, d=128, page=64)
    table = b.table.clone()
    for s in (1, 2):
        table[s, :10] = table[0, :10]
        b.k[s][:640], b.v[s][:640] = b.k[0][:640], b.v[0][:640]
    b.table = table
    o, lse = b.run(b.plan())
    b.check(o, lse)


def test_nothing_to_do():
    b = Batch(seed=15, new=[0, 0], ctx=[5, 0], heads=2, kv=1, d=64, page=32, pad=3)
    plan = b.plan()
    o, lse = b.run(plan)
    b.check(o, lse)
    empty = torch.empty(0, 2, 64, dtype=BF, device="cuda")
    plan.rf2_paged_attn(empty, b.k_cache, b.v_cache, b.table, b.seq_len, b.cu, plan.alloc_workspace(), empty)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    plan.rf2_paged_attn(b.q, b.k_cache, b.v_cache, none, none, none.new_zeros(1), plan.alloc_workspace(), o)
    torch.cuda.synchronize()
    assert (o == 7.0).all()
