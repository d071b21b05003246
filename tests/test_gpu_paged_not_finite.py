"""Values of V that are not finite, where a tile's rows all belong to one token and in the first units that a row sees; large ones."""
import pytest
import torch

from tests.paged_ref import Batch, attention, put_many

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")


def set_v(b, s, pos, ch, x):
    """Channel ch of V of token pos of sequence s, all K/V heads."""
    page, r = int(b.table[s, pos // b.page]), pos % b.page
    b.v_cache[page, :, r // 32, r % 32 // 16 * 2 + r % 8 // 4, ch, r % 16 // 8 * 4 + r % 4] = x


def bits(x):
    return x.contiguous().view(torch.int16)


# rows of a token that fill whole tiles of 16, of 32 and of a wavefront's 64: the rows of a tile then all see the same keys, and the tokens
# behind stand in the same unit of 32 keys
@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads, new, ctx", [(16, [2, 0], [40, 0]), (16, [4, 0, 0, 0], [0, 9, 0, 3]), (32, [2, 0], [100, 5]), (40, [3, 0, 0, 0], [70, 0, 0, 0]),
                                             (64, [7], [40]), (64, [30, 2], [900, 0]), (128, [9], [0]), (100, [11], [33]), (512, [5], [3])], ids=str)
def test_one_token_to_a_tile(heads, new, ctx, d, dtype):
    b = Batch(seed=30, new=new, ctx=ctx, heads=heads, kv=1, d=d, page=64, dtype=dtype)
    plan = b.plan()
    n, last = new[0], ctx[0] + new[0] - 1
    values = [(0, INF), (1, -INF), (2, NAN), (d - 1, NAN)]
    for first in {1, n // 2, n - 1}:                       # tokens from this one on
        spots = range(ctx[0] + first, last + 1)
        for ch, _ in values:
            for pos in spots:
                set_v(b, 0, pos, ch, 0.0)
        clean, _ = b.run(plan)
        for ch, x in values:
            for pos in spots:
                set_v(b, 0, pos, ch, x)
        o, _ = b.run(plan)
        for ch, _ in values:
            for pos in spots:
                set_v(b, 0, pos, ch, 0.0)
        assert torch.equal(bits(o[:first]), bits(clean[:first])), first
        assert torch.equal(bits(o[first:, :, 3:d - 1]), bits(clean[first:, :, 3:d - 1])), first
        seen = o[first:n].float()
        assert (seen[:, :, 0] == INF).all() and (seen[:, :, 1] == -INF).all() and torch.isnan(seen[:, :, [2, d - 1]]).all(), first


# a chunk whose partial last unit stands in the same wavefront's list as the unit with the values, which comes right behind it
@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new, ctx, heads, kv", [([60], [5], 1, 1), ([70], [16], 1, 1), ([61], [0], 2, 1), ([45, 50], [3, 20], 4, 2), ([40], [60], 1, 1),
                                                 ([130], [7], 3, 1)], ids=str)
def test_an_infinite_value_reaches_every_row_that_sees_it(new, ctx, heads, kv, d, dtype):
    b = Batch(seed=31, new=new, ctx=ctx, heads=heads, kv=kv, d=d, page=64, dtype=dtype)
    plan = b.plan()
    for t in (0, 5, 33):                                   # a token of the chunks
        at = 0
        for s, n in enumerate(new):
            for ch in (0, 1):
                set_v(b, s, ctx[s] + t, ch, 0.0)
        clean, _ = b.run(plan)
        for s, n in enumerate(new):
            set_v(b, s, ctx[s] + t, 0, INF)
            set_v(b, s, ctx[s] + t, 1, -INF)
        o, _ = b.run(plan)
        for s, n in enumerate(new):
            got, want = o[at:at + n], clean[at:at + n]
            assert torch.equal(bits(got[:t]), bits(want[:t])), (t, s)
            assert torch.equal(bits(got[:, :, 2:]), bits(want[:, :, 2:])), (t, s)
            assert (got[t:, :, 0].float() == INF).all() and (got[t:, :, 1].float() == -INF).all(), (t, s)
            for ch in (0, 1):
                set_v(b, s, ctx[s] + t, ch, b.v[s][ctx[s] + t, 0, ch].item())
            at += n


@pytest.mark.parametrize("dtype, size", [(torch.bfloat16, 2.0 ** 64), (torch.float16, 2.0 ** 13)], ids=["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[1, 1], [70, 3]], ids=["few", "many"])
def test_large_values_stay_finite(new, d, dtype, size):
    """V of up to 2^67 in bf16 (nearly all of fp16), behind logits that grow by 38 octaves, so that references lag."""
    b = Batch(seed=32, new=new, ctx=[640, 300], heads=2, kv=1, d=d, page=32, dtype=dtype)
    b.q.zero_()
    b.q[:, :, 0] = 1.0
    for s in (0, 1):
        b.k[s] = torch.zeros(b.len[s], 1, d)
        b.k[s][:, 0, 0] = torch.linspace(0, 38 * 0.6931 * d ** 0.5, b.len[s])
        b.k[s] = b.k[s].to(dtype)
        b.v[s] = (b.v[s].double().clamp(-7.9, 7.9) * size).to(dtype)
        pos = torch.arange(b.len[s])
        slots = b.table[s].cpu()[pos // 32].long() * 32 + pos % 32
        k_cache, v_cache = b.k_cache.cpu(), b.v_cache.cpu()
        put_many(k_cache, v_cache, slots, b.k[s], b.v[s], 32)
        b.k_cache.copy_(k_cache)
        b.v_cache.copy_(v_cache)
    o, lse = b.run(b.plan())
    at = 0
    for s, n in enumerate(new):
        want, want_lse, tol, lse_tol = attention(b.q[at:at + n], b.k[s].cuda(), b.v[s].cuda(), b.kept[s].cuda(), n, True, d ** -0.5, torch.finfo(dtype).eps / 2)
        # (logits up to 27 in place of 8: 2^-18 of a probability more, twice)
        assert ((o[at:at + n].double() - want).abs() <= tol + 2.0 ** -17 * b.v[s].abs().max().item()).all()
        assert ((lse[at:at + n].double() - want_lse).abs() <= lse_tol + 2.0 ** -17).all()
        at += n
