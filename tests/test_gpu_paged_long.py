"""Attention of chunks with more tiles of rows than the workspace has places for, against its definition in 64 bits."""
import pytest
import torch

from tests.paged_ref import Batch, attention

pytestmark = pytest.mark.gpu

CASES = {
    "one_tile_more": dict(new=[4097], ctx=[0], heads=32, kv=1, d=64, page=256),
    "prompt": dict(new=[5000], ctx=[300], heads=32, kv=1, d=64, page=64, dtype=torch.float16, pad=3),
    "prompt_d128": dict(new=[4500], ctx=[0], heads=32, kv=1, d=128, page=128),
    "prompts": dict(new=[2700, 2, 1500, 2100], ctx=[0, 900, 40, 0], heads=64, kv=2, d=64, page=128),
    # a long sequence that is cut, before one that is not
    "cut_before_whole": dict(new=[3200, 7360], ctx=[100000, 0], heads=32, kv=8, d=128, page=256),
    # before more sequences than a wavefront has lanes
    "before_many": dict(new=[4200] + [1] * 64 + [0, 3], ctx=[0] * 40 + [70] * 27, heads=32, kv=1, d=64, page=64),
    "before_many_d128": dict(new=[4200] + [0] * 100 + [5] * 30, ctx=[0] * 131, heads=32, kv=1, d=128, page=64, dtype=torch.float16),
}


@pytest.mark.parametrize("name", list(CASES))
def test_chunks_of_many_tiles(name):
    b = Batch(seed=40, **CASES[name])
    for causal in (True, False) if name == "one_tile_more" else (True,):
        plan = b.plan(causal)
        o, lse = b.run(plan)
        share = b.check(o, lse, causal)
        print(f"{name} causal={causal}: {share:.3f} of the tolerance")
        o2, _ = b.run(plan, with_lse=False)
        assert torch.equal(o.view(torch.int16), o2.view(torch.int16)), "the same call, the same bits"


@pytest.mark.parametrize("heads, new", [(16, [2200] + [0, 1] * 900 + [0] * 2295), (32, [1100] + [0, 1] * 1400 + [0] * 1295)], ids=["16_rows", "32_rows"])
def test_a_long_chunk_among_thousands_of_sequences(heads, new):
    """Few rows a sequence on average: tiles of 16 and of 32 rows, 2,200 and 1,100 of them of one sequence."""
    b = Batch(seed=41, new=new, ctx=[0] * len(new), heads=heads, kv=1, d=64, page=32)
    o, lse = b.run(b.plan())
    n = new[0]
    want, want_lse, tol, lse_tol = attention(b.q[:n], b.k[0].cuda(), b.v[0].cuda(), b.kept[0].cuda(), n, True, 0.125, 2.0 ** -8)
    assert ((o[:n].double() - want).abs() <= tol).all() and ((lse[:n].double() - want_lse).abs() <= lse_tol).all()
    # one key each: its row of V
    ones = torch.cat([b.v[s] for s in range(1, len(new)) if new[s]]).cuda()
    assert ones.shape[0] == sum(new) - n and torch.equal(o[n:], ones.expand(-1, heads, -1))
